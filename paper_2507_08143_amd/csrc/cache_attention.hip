// Attention of new tokens to a paged cache (see compactor_cache_attention).
//
// A step reads every cached row once and multiplies it with the few query rows of its head (the G query heads of T new
// tokens): 512 bytes a slot against 512 G T flops, so it is bound by HBM for all G T <= 64.  What carries it is that
// nothing stands between the loads: both products take the rows as they arrive in registers, without LDS.
//
// A wave takes tiles of 32 slots.  S^T = K Q^T (16x16x32 MFMA, twice): a lane holds row l & 15 of a half of the tile in
// 16-byte pieces (channels 32 kk + 8 (l >> 4) ..), which is the A operand as it stands, and gets logits of query l & 15 and
// slots 4 (l >> 4) + v of each half.  For O^T = V^T P^T the contraction runs over slots, in an order that is free as long as
// both operands have the same: lane group l >> 4 takes the slots whose logits it has, so P needs no exchange, and loads
// those 8 rows of V, piece l & 15 of each: whole rows per 16 lanes.  8 rows x 8 channels of a lane, transposed in place by 32
// byte permutations, are the A operands of eight MFMAs; the c-th has channel 8 (l & 15) + c in its row l & 15, which leaves lane l
// with channels 32 (l >> 4) .. + 32 of query l & 15: the query whose maximum and sum it has, and consecutive.
//
// The length of a head is split over workgroups, and over the four waves of each; the waves meet in LDS, the workgroups
// in a second launch (attend_join_kernel), which also adds the weights to the mass: they are only known once the sum is, so the logits
// wait in the workspace, 4 bytes a slot and query row, or a third launch has K again (attend_mass_kernel).
#include <type_traits>

#include "attend.h"

namespace cmp {

// Two weights as sums of three bf16 numbers, 8 bits of their 24 each: truncated, so that no number is negative, and the two smaller ones no
// less than 2^-126 unless the weight is 0.  A row of V with an infinity then adds infinities of one sign (with a difference of rounded numbers,
// or 0 times it, their sum is NaN).  x: 0 or at least 2^-126.  (us with two rounded planes, 16 bits / with three: 2.3 M slots, 4 rows 248 / 249; 96 heads
// of 18000, 32 rows 184 / 186, 40 rows with weights 302 / 313, 64 rows 230 / 260.)
__device__ __forceinline__ void split(float x0, float x1, unsigned &hi, unsigned &mid, unsigned &lo) {
  const auto rest = [](float x, float least) { return fmaxf(x - __uint_as_float(__float_as_uint(x) & 0xffff0000u), least); };
  const auto upper = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
  const float least0 = fminf(x0, 0x1p-126f), least1 = fminf(x1, 0x1p-126f);
  hi = upper(x0, x1);
  x0 = rest(x0, least0);
  x1 = rest(x1, least1);
  mid = upper(x0, x1);
  lo = upper(rest(x0, least0), rest(x1, least1));
}

// Where the rows of a wave's tiles lie.  PAGE16: pages hold whole halves of tiles, so a half has one origin, the same for all
// lanes; lane i keeps that of half i & 1 of tile i >> 1 of a run of 32, and a tile reads its two from there.  Else lane i keeps
// the origin of slot i & 31 of the next tile, with the page of the one after on its way.
template <bool PAGE16>
struct Places {
  long long off;               // elements, of the lane's half (slot)
  unsigned long long there;    // bit i: what lane i stands for holds a token
  int page, at;                // !PAGE16: the tile after the next
  bool in;
};

template <bool PAGE16>
__device__ __forceinline__ void places_run(const CacheView &C, const HeadPlace &p, int first, int count, int lane, Places<PAGE16> &P) {
  // PAGE16: halves of the tiles from `first` on
  const long long slot = (long long)first + 16 * lane;
  bool ok = slot < count;
  const int i = invariant_quotient(ok ? (unsigned)slot : 0u, C.div_mul, C.div_shift);
  const int page = ok ? p.table[i] : 0;
  ok = ok && page_there(C, page);
  P.off = ok ? page * C.page_stride + ((int)slot - i * C.page_size) * C.slot_stride : 0;
  P.there = __ballot(ok);
}
template <bool PAGE16>
__device__ __forceinline__ void places_fetch(const CacheView &C, const HeadPlace &p, long long first, int count, int lane, Places<PAGE16> &P) {
  const long long slot = first + (lane & 31);
  P.in = slot < count;
  const int i = invariant_quotient(P.in ? (unsigned)slot : 0u, C.div_mul, C.div_shift);
  P.page = P.in ? p.table[i] : 0;
  P.at = (int)slot - i * C.page_size;
}
template <bool PAGE16>
__device__ __forceinline__ void places_take(const CacheView &C, Places<PAGE16> &P) {
  const bool ok = P.in && page_there(C, P.page);
  P.off = ok ? P.page * C.page_stride + P.at * C.slot_stride : 0;
  P.there = __ballot(ok);
}

// K or V rows of a tile.  K: pieces 4 kk + (l >> 4) of rows l & 15 of both halves.  V: piece l & 15 of rows 4 (l >> 4) + i of both.
// lane_at (PAGE16): the lane's place in a half, bytes; stride: of a slot, bytes.
template <bool PAGE16, bool K>
__device__ __forceinline__ void load_rows(const uint16_t *base, const Places<PAGE16> &P, int tile, int lane, unsigned lane_at, unsigned stride, Piece (&x)[8]) {
  if (PAGE16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const char *half = reinterpret_cast<const char *>(base + from_lane(P.off, 2 * tile + (i >> 2)));
      const char *at = (K ? half + 64 * (i & 3) : half + (i & 3) * (long long)stride) + lane_at;
      // (the two halves of a 128-byte line of K are read by two instructions: streaming, the second would miss again)
      x[i].u = K ? *reinterpret_cast<const uint4 *>(at) : load_stream16(at);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long long off = __shfl(P.off, 16 * (i >> 2) + (K ? lane & 15 : 4 * (lane >> 4) + (i & 3)));
      const uint16_t *at = base + off + (K ? 8 * (lane >> 4) + 32 * (i & 3) : 8 * (lane & 15));
      x[i].u = K ? *reinterpret_cast<const uint4 *>(at) : load_stream16(at);
    }
  }
}

// Logits leave for the workspace 16 bytes a lane, or by way of LDS in whole lines, a run of tiles of a row at a time; up to 16 rows that pays
// (with weights in 16 bits: 2.3 M slots with 4 rows: 249 us and 255, without logits 221; streamed, or behind the last barrier: the same), with 20 rows 66 us and 64, with 40 158 and 102.
constexpr int KEPT_FLOATS = 2048;            // that a wave keeps: 4 tiles of 16 rows
template <int NT> constexpr bool kept_in_lds = NT == 1;
template <int NT>
struct AttendLds {
  float o[ATT_WAVES][16][D + 4];
  float kept[ATT_WAVES][kept_in_lds<NT> ? KEPT_FLOATS : 4], p[ATT_WAVES][16][ATT_TILE + 1];
  float m[ATT_WAVES][16 * NT], l[ATT_WAVES][16 * NT];
  float lse2[16 * NT];
  int none;
};

template <int NT, bool PAGE16>
__global__ __launch_bounds__(256, NT <= 2 ? 2 : 1) void attend_kernel(const CacheView C, const Queries Q) {
  __shared__ AttendLds<NT> L;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, j = lane >> 4;
  const int R = Q.tokens * Q.group;
  Fragment part;
  int fragment = (int)blockIdx.x;
  if (!(Q.target > 0 ? scan_part(C, Q, fragment, part) : split_part(C, Q, part, fragment))) {
    if (tid == 0) Q.frags[fragment].head = -1;
    return;
  }
  if (Q.frags != nullptr && tid == 0) {
    Q.frags[fragment] = part;
    if (Q.head_frags != nullptr && part.step0 == 0) Q.head_frags[part.head] = make_int2(part.first, part.parts);
  }
  const unsigned g = (unsigned)part.head;
  const HeadOf w = head_of(C, g);
  const HeadPlace hp = head_place(C, w);
  const int count = part.count, n = part.n;
  const bool complete = part.parts == 1;
  if (tid == 0) L.none = 0;
  const Run run = run_of(part, wave);
  const int first = run.first, tiles = run.tiles;
  const int seen_by_all = count - (n - 1);
  const uint16_t *kp = C.k + hp.rows, *vp = C.v + hp.rows;

  Places<PAGE16> P;
  if (PAGE16) {
    places_run(C, hp, first, count, lane, P);
  } else {
    places_fetch(C, hp, first, count, lane, P);
    places_take(C, P);
    places_fetch(C, hp, (long long)first + ATT_TILE, count, lane, P);
  }
  Piece q[NT][4];
  int see[NT];
  load_queries<NT>(Q, w, R, count, n, q, see);
  Piece k[8], v[8];
  const unsigned stride = PAGE16 ? 2u * (unsigned)C.slot_stride : 0u, k_at = n16 * stride + 16 * j, v_at = 4 * j * stride + 16 * n16;
  auto tile_there = [&](int tile) {
    if (!PAGE16) return (unsigned)P.there;
    const unsigned two = (unsigned)(P.there >> (2 * (tile & 31)));
    return (two & 1u ? 0xffffu : 0u) | (two & 2u ? 0xffff0000u : 0u);
  };
  f32x4 acc[NT][8];
  float m[NT], l[NT];            // of query l & 15: reference of its exponents, the lane's part of their sum
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    l[nt] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[nt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const Scaling scaling = scaling_of(Q);
  const bool store = Q.logits != nullptr && count <= Q.most;
  float *logits = Q.logits + (long long)g * R * Q.pitch;
  float *kept = L.kept[wave];
  const int kept_tiles = kept_in_lds<NT> ? KEPT_FLOATS / (ATT_TILE * R) : 1;
  auto leave = [&](int upto) {              // tiles up to this one
    wave_lds_fence();
    const int t0 = (upto - 1) / kept_tiles * kept_tiles, quads = (upto - t0) * (ATT_TILE / 4);
    for (int row = 0; row < R; ++row)
      for (int u = lane; u < quads; u += 64)
        *reinterpret_cast<f32x4 *>(logits + (long long)row * Q.pitch + first + t0 * ATT_TILE + 4 * u) =
            *reinterpret_cast<const f32x4 *>(kept + ((u >> 3) * R + row) * ATT_TILE + 4 * (u & 7));
    wave_lds_fence();
  };

  unsigned there;                // bit i: slot i of the tile holds a token whose page is there
  auto one_tile = [&](int tile, auto another) {
    constexpr bool more = decltype(another)::value;
    const int s0 = first + tile * ATT_TILE;
    f32x4 s[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        s[nt][half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          s[nt][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[4 * half + kk].v, q[nt][kk].v, s[nt][half], 0, 0, 0);
      }
    // K of the next tile leaves as soon as its registers are free, V after the second product.
    unsigned there_next = 0;
    if constexpr (more) {
      if (PAGE16) {
        if (((tile + 1) & 31) == 0) places_run(C, hp, s0 + ATT_TILE, count, lane, P);
      } else {
        places_take(C, P);
        places_fetch(C, hp, (long long)s0 + 2 * ATT_TILE, count, lane, P);
      }
      load_rows<PAGE16, true>(kp, P, (tile + 1) & 31, lane, k_at, stride, k);
      there_next = tile_there(tile + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int left = count - s0;
    if (left < 32) there &= (1u << left) - 1u;              // left >= 1
    const bool whole = there == 0xffffffffu && s0 + ATT_TILE <= seen_by_all;      // the same for all lanes
    const unsigned there_at = there >> (4 * j);             // bit 16 (i >> 2) + (i & 3): the lane's i-th slot
    bool ahead = false;
    if (__builtin_expect(!whole, 0)) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned keep = there_at >> (16 * (i >> 2) + (i & 3)) & 1u ? 0xffffffffu : 0u;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          v[i].w[d] &= keep;
          odd |= (v[i].w[d] & 0x7f80u) == 0x7f80u || (v[i].w[d] & 0x7f800000u) == 0x7f800000u;
        }
      }
      // The row of a later token is no part of an earlier one's output even where it holds no number (0 * inf).  Where such a tile
      // has any, the rows that not all queries see are left out of the product and added one by one.
      if (s0 + ATT_TILE > seen_by_all && __any(odd)) {
        ahead = true;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const unsigned keep = s0 + 4 * j + 16 * (i >> 2) + (i & 3) < seen_by_all ? 0xffffffffu : 0u;
#pragma unroll
          for (int d = 0; d < 4; ++d) v[i].w[d] &= keep;
        }
      }
    }
    Piece hi[NT], mid[NT], lo[NT];          // P as three bf16 planes, B operands: split()
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
      if (scaling.capped) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = capped_logit(scaling, s[nt][i >> 2][i & 3]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[nt][i >> 2][i & 3] * scaling.to_base2;
      }
      if (__builtin_expect(!whole, 0)) {
        const int upto = see[nt] - s0 - 4 * j;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int at = 16 * (i >> 2) + (i & 3);
          x[i] = (there_at >> at & 1u) && at < upto ? x[i] : -INFINITY;
        }
      }
      if (store && 16 * nt + n16 < R) {
        float *to = (kept_in_lds<NT> ? kept + ((tile % kept_tiles) * R + n16) * ATT_TILE : logits + (long long)(16 * nt + n16) * Q.pitch + s0) + 4 * j;
        *reinterpret_cast<f32x4 *>(to) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4 *>(to + 16) = f32x4{x[4], x[5], x[6], x[7]};
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
      top = quarters_max(top);
      // the reference moves only when it has fallen 2^8 behind: weights up to 2^8 keep their precision
      if (__any(top > m[nt] + 8.f)) {
        const float to = fmaxf(m[nt], top), f = to == -INFINITY ? 1.f : exp2_(m[nt] - to);
        m[nt] = to;
        l[nt] *= f;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[nt][c] *= f;
      }
      const float ref = m[nt] == -INFINITY ? 0.f : m[nt];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = exp2_(x[i] - ref);
        sum += x[i];
      }
      l[nt] += sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) split(x[2 * i], x[2 * i + 1], hi[nt].w[i], mid[nt].w[i], lo[nt].w[i]);
      if (__builtin_expect(ahead, 0)) {
        float *mine = L.p[wave][n16];
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 8; ++i) mine[16 * (i >> 2) + 4 * j + (i & 3)] = x[i];
        wave_lds_fence();
#pragma unroll 1
        for (int i = max(seen_by_all - s0, 0); i < min(left, ATT_TILE); ++i) {
          if (!(there >> i & 1u)) continue;
          const long long row = row_at(C, hp, slot_place(C, hp, s0 + i));
          if (s0 + i >= see[nt]) continue;
          const float weight = mine[i];
#pragma unroll
          for (int vv = 0; vv < 4; ++vv) {
            Piece y;
            y.u = *reinterpret_cast<const uint4 *>(C.v + row + 32 * j + 8 * vv);
#pragma unroll
            for (int c = 0; c < 8; ++c)
              acc[nt][c][vv] = fmaf(weight, __uint_as_float(c & 1 ? y.w[c >> 1] & 0xffff0000u : y.w[c >> 1] << 16), acc[nt][c][vv]);
          }
        }
      }
    }
    if (kept_in_lds<NT> && store && more && (tile + 1) % kept_tiles == 0) leave(tile + 1);
    // channels 2 d and 2 d + 1 of the lane's piece, 8 slots each
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      Piece a;
#pragma unroll
      for (int i = 0; i < 4; ++i) a.w[i] = __builtin_amdgcn_perm(v[2 * i + 1].w[c >> 1], v[2 * i].w[c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        acc[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, hi[nt].v, acc[nt][c], 0, 0, 0);
        acc[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, mid[nt].v, acc[nt][c], 0, 0, 0);
        acc[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, lo[nt].v, acc[nt][c], 0, 0, 0);
      }
    }
    if constexpr (more) load_rows<PAGE16, false>(vp, P, (tile + 1) & 31, lane, v_at, stride, v);
    there = there_next;
    __builtin_amdgcn_sched_barrier(0);
  };
  // No load of rows of the loop is under a condition, or the compiler would have to wait for V where it waits for K; nor is one
  // issued that nobody wants: the barrier below would wait for it.
  if (tiles > 0) {
    load_rows<PAGE16, true>(kp, P, 0, lane, k_at, stride, k);
    load_rows<PAGE16, false>(vp, P, 0, lane, v_at, stride, v);
    there = tile_there(0);
    for (int tile = 0; tile + 1 < tiles; ++tile) one_tile(tile, std::true_type());
    one_tile(tiles - 1, std::false_type());
  }

  waves_meet<NT>(C, Q, w, part, fragment, L, acc, m, l, see);
  if (kept_in_lds<NT> && store && tiles > 0) leave(tiles);
  if (complete && store && n > 0) mass_here(C, Q, hp, logits, R, count, L.lse2, &L.none);
}

// A query row of a head's fragments, all of its channels: SIDE fragments side by side, 8 channels a thread.
template <int SIDE>
__device__ __forceinline__ void join_fragments(const Queries &Q, int2 f, int R, int r, const float2 &all, int sl, int ch, f32x4 (&o)[2]) {
  o[0] = o[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll SIDE < 16 ? 4 : 1
  for (int k = sl; k < f.y; k += SIDE) {
    const long long at = (long long)(f.x + k) * R + r;
    const float mk = Q.stats[at].x, scale = all.x == -INFINITY ? 0.f : exp2_(mk - all.x);
    const f32x4 *x = reinterpret_cast<const f32x4 *>(Q.partial + at * D + ch);
    o[0] += x[0] * scale;
    o[1] += x[1] * scale;
  }
}

// Second launch: the fragments of a head meet.  The first workgroups take a query row each, 16 fragments side by side and 8 channels a thread, or (WAVES)
// four, a wave each with 4 fragments side by side; the others add a fragment's weights to the mass.
template <bool WAVES>
__global__ __launch_bounds__(256) void attend_join_kernel(const CacheView C, const Queries Q) {
  __shared__ float part_o[WAVES ? 1 : 16][D + 4], lse2[MOST_ROWS];
  __shared__ float2 stats[256];                     // of the groups of more than 16 rows
  __shared__ int none;
  const int tid = threadIdx.x, R = Q.tokens * Q.group;
  const unsigned rows = (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads * (unsigned)R;
  const unsigned blocks = WAVES ? (rows + 3) / 4 : rows;
  if (blockIdx.x < blocks) {
    const unsigned at = WAVES ? 4 * blockIdx.x + (unsigned)__builtin_amdgcn_readfirstlane(tid >> 6) : blockIdx.x;
    if (at >= rows) return;
    const unsigned g = at / (unsigned)R;
    const int r = (int)(at - g * (unsigned)R);
    const int2 f = Q.head_frags[g];
    if (f.y < 2) return;                            // its only workgroup has finished it
    const float2 all = join_stats(Q, f.x, f.y, R, r);      // (every wave)
    const int sl = WAVES ? tid >> 4 & 3 : tid >> 4, ch = 8 * (tid & 15);
    f32x4 o[2];
    join_fragments<WAVES ? 4 : 16>(Q, f, R, r, all, sl, ch, o);
    if (WAVES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i >> 2][i & 3] = quarters_sum(o[i >> 2][i & 3]);
      if (sl == 0) finish_row(C, Q, head_of(C, g), r, ch, o, all.x, all.y);
      return;
    }
    *reinterpret_cast<f32x4 *>(&part_o[sl][ch]) = o[0];
    *reinterpret_cast<f32x4 *>(&part_o[sl][ch + 4]) = o[1];
    __syncthreads();
    if (tid < 16) {
      o[0] = o[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        o[0] += *reinterpret_cast<const f32x4 *>(&part_o[s][ch]);
        o[1] += *reinterpret_cast<const f32x4 *>(&part_o[s][ch + 4]);
      }
      finish_row(C, Q, head_of(C, g), r, ch, o, all.x, all.y);
    }
    return;
  }
  const Fragment f = Q.frags[blockIdx.x - blocks];
  if (f.head < 0 || f.parts < 2 || f.count > Q.most) return;
  const HeadPlace hp = head_place(C, head_of(C, (unsigned)f.head));
  const float *logits = Q.logits + (long long)f.head * R * Q.pitch;
  const int from = f.step0 * ATT_STEP, to = min(f.step1 * ATT_STEP, f.count);
  if (from >= to) return;
  if (tid == 0) none = 0;
  __syncthreads();
  MassQuad M;
  mass_fetch(C, Q, hp, logits, R, min(from + 4 * tid, (to - 1) & ~3), to, M);
  row_sums(Q, f, R, stats, lse2, &none);
  __syncthreads();
  for (int at = from + 4 * tid; at < to; at += 4 * 256) {
    if (at >= from + 4 * 256) mass_fetch(C, Q, hp, logits, R, at, to, M);
    mass_add(Q, lse2, none, logits, R, at, M);
  }
}

// Where there are many rows each has few fragments, and what counts is how many workgroups start: for rows of 4 bits, where that is a larger part of a call, a
// wave a row from this many on (us with a workgroup a row / a wave: 96 heads of 900 to 9831, 20 rows with their mass 44.3 / 41.9; 1024 of 500 to 4000, 4 rows
// 89.0 / 83.6; 192 of 8192 to 32000, 40 rows 286 / 278; but 8 of 8000, 7 rows, 13.4 / 15.3, of 32000 20.6 / 26.2).
constexpr long long JOIN_WAVES = 1024;

// Weights of many rows from K, which is read again: 256 bytes a slot, where the logits' way through the workspace takes 8 for every row.
// (Third launch.)  A fragment a workgroup; its rows' sums are known.  A lane has 8 slots of query l & 15 as in attend_kernel, and the sum over the
// rows is one over its tiles of rows and 16 lanes.
template <int NT, bool PAGE16>
__global__ __launch_bounds__(256) void attend_mass_kernel(const CacheView C, const Queries Q) {
  __shared__ float2 stats[256];
  __shared__ float lse2[MOST_ROWS];
  __shared__ int none;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, j = lane >> 4;
  const int R = Q.tokens * Q.group;
  const Fragment part = Q.frags[blockIdx.x];
  if (part.head < 0 || part.n <= 0 || part.count > Q.most) return;
  if (tid == 0) none = 0;
  __syncthreads();
  const HeadOf w = head_of(C, (unsigned)part.head);
  const HeadPlace hp = head_place(C, w);
  const int count = part.count, seen_by_all = count - (part.n - 1);
  const Run run = run_of(part, wave);
  const int first = run.first, tiles = run.tiles;
  const uint16_t *kp = C.k + hp.rows;
  Places<PAGE16> P;
  if (PAGE16) {
    places_run(C, hp, first, count, lane, P);
  } else {
    places_fetch(C, hp, first, count, lane, P);
    places_take(C, P);
    places_fetch(C, hp, (long long)first + ATT_TILE, count, lane, P);
  }
  Piece q[NT][4], k[8];
  int see[NT];
  load_queries<NT>(Q, w, R, count, part.n, q, see);
  const unsigned stride = PAGE16 ? 2u * (unsigned)C.slot_stride : 0u, k_at = n16 * stride + 16 * j;
  auto tile_there = [&](int tile) {
    if (!PAGE16) return (unsigned)P.there;
    const unsigned two = (unsigned)(P.there >> (2 * (tile & 31)));
    return (two & 1u ? 0xffffu : 0u) | (two & 2u ? 0xffff0000u : 0u);
  };
  unsigned there = 0;
  if (tiles > 0) {
    load_rows<PAGE16, true>(kp, P, 0, lane, k_at, stride, k);
    there = tile_there(0);
  }
  row_sums(Q, part, R, stats, lse2, &none);
  __syncthreads();
  float z[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) z[nt] = see[nt] > 0 ? lse2[16 * nt + n16] : INFINITY;
  const Scaling scaling = scaling_of(Q);
  float *weights = Q.weights + (long long)part.head * Q.pitch;

  auto one_tile = [&](int tile, auto another) {
    constexpr bool more = decltype(another)::value;
    const int s0 = first + tile * ATT_TILE;
    f32x4 s[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        s[nt][half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          s[nt][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[4 * half + kk].v, q[nt][kk].v, s[nt][half], 0, 0, 0);
      }
    unsigned there_next = 0;
    if constexpr (more) {
      if (PAGE16) {
        if (((tile + 1) & 31) == 0) places_run(C, hp, s0 + ATT_TILE, count, lane, P);
      } else {
        places_take(C, P);
        places_fetch(C, hp, (long long)s0 + 2 * ATT_TILE, count, lane, P);
      }
      load_rows<PAGE16, true>(kp, P, (tile + 1) & 31, lane, k_at, stride, k);
      there_next = tile_there(tile + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int left = count - s0;
    if (left < 32) there &= (1u << left) - 1u;
    const bool whole = there == 0xffffffffu && s0 + ATT_TILE <= seen_by_all;
    const unsigned there_at = there >> (4 * j);
    float sum[8] = {};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
      if (scaling.capped) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = capped_logit(scaling, s[nt][i >> 2][i & 3]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[nt][i >> 2][i & 3] * scaling.to_base2;
      }
      if (__builtin_expect(!whole, 0)) {
        const int upto = see[nt] - s0 - 4 * j;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int at = 16 * (i >> 2) + (i & 3);
          x[i] = (there_at >> at & 1u) && at < upto ? x[i] : -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += z[nt] == INFINITY ? 0.f : exp2_(x[i] - z[nt]);
    }
    const float mine = lanes_sum(sum, n16);
    if (n16 < 8) weights[s0 + 16 * (n16 >> 2) + 4 * j + (n16 & 3)] = mine;
    there = there_next;
    __builtin_amdgcn_sched_barrier(0);
  };
  if (tiles > 0) {
    for (int tile = 0; tile + 1 < tiles; ++tile) one_tile(tile, std::true_type());
    one_tile(tiles - 1, std::false_type());
  }
  weights_to_mass(C, Q, hp, weights, run, &none);
}

static float scale_of(const compactor_cache_query_t *q) { return q->scale > 0.f ? q->scale : 1.0f / sqrtf((float)D); }

static int query_check(const compactor_cache_query_t *q, const CacheView &C) {
  if (!q) return COMPACTOR_EINVAL;
  if (q->tokens < 1 || q->q_heads < C.kv_heads || q->q_heads % C.kv_heads || q->max_tokens < 0) return COMPACTOR_EINVAL;
  if ((long long)(q->q_heads / C.kv_heads) * q->tokens > 64) return COMPACTOR_EUNSUPPORTED;
  // (in base 2 too, and relative to the cap)
  if (!(q->scale >= 0.f) || !isfinite(q->scale * LOG2E) || !(q->softcap >= 0.f) || !isfinite(q->softcap * LOG2E)) return COMPACTOR_EINVAL;
  if (q->softcap > 0.f && !isfinite(scale_of(q) / q->softcap)) return COMPACTOR_EINVAL;
  return COMPACTOR_OK;
}

static int query_most(const CacheView &C, const compactor_cache_query_t *q) {
  return q->max_tokens > 0 && q->max_tokens < C.capacity ? q->max_tokens : C.capacity;
}

struct AttendPlan {
  int rows, frags_most, target, split, pitch;
  bool joined;                 // heads may have several fragments
  bool again;                  // weights from K, read again
  size_t frags, head_frags, partial, stats, logits;       // bytes, in this order in the workspace (logits: or weights)
  size_t bytes() const { return frags + head_frags + partial + stats + logits; }
};

static AttendPlan attend_plan(const CacheView &C, const compactor_cache_query_t *q, const AttendKernels &kernels) {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    cus = 256;
  AttendPlan A;
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads, most = query_most(C, q);
  const long long steps = (most + ATT_STEP - 1) / ATT_STEP;
  A.rows = q->tokens * (q->q_heads / C.kv_heads);
  A.split = 1;
  A.target = A.frags_most = 0;
  // a wave adds up the steps of heads that may hold more than `most`, and their fragments have to fit all the same
  if (steps > ATT_ALONE && heads <= SCAN_HEADS && heads * (((long long)C.capacity + ATT_STEP - 1) / ATT_STEP) <= 0x7fffffffll) {
    A.target = kernels.bits4 ? bits4_fragment_target(heads, steps, A.rows, cus, C.slot_stride > ROW4) : fragment_target(heads, steps, A.rows, cus);
    A.frags_most = fragments_most((int)heads, A.target);
  } else if (steps > ATT_ALONE) {
    A.split = (int)std::max(std::min(std::min(SPLIT_ALL / heads, (long long)SPLIT_MOST), ((steps - 1) >> ATT_LEAST_LOG) + 1), 1ll);
    if (A.split > 1) A.frags_most = A.split * (int)heads;
  }
  A.joined = A.frags_most > 0;
  A.pitch = (int)((most + ATT_TILE - 1) / ATT_TILE * ATT_TILE);
  const size_t a_row = (size_t)heads * A.pitch * sizeof(float);
  A.again = q->accumulate && A.rows > kernels.again_rows && a_row * A.rows > kernels.again_bytes;
  if (A.again && A.frags_most == 0) A.frags_most = (int)heads;        // one each, for what is known of them
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  const size_t n = A.frags_most;
  A.frags = up(n * sizeof(Fragment));
  A.head_frags = A.joined ? up((size_t)heads * sizeof(int2)) : 0;
  A.partial = A.joined ? up(n * A.rows * D * sizeof(float)) : 0;
  A.stats = up(n * A.rows * sizeof(float2));
  A.logits = q->accumulate ? up(A.again ? a_row : a_row * A.rows) : 0;
  return A;
}

template <bool PAGE16>
static void launch_attend(const CacheView &C, const Queries &Q, unsigned blocks, hipStream_t st) {
  // tiles of 16 query rows (40 rows, 96 heads of 18000: 208 us with three, 240 with four; 24 of them 62 and 72)
  const int rows = Q.tokens * Q.group;
  const auto kernel = rows <= 16   ? attend_kernel<1, PAGE16>
                      : rows <= 32 ? attend_kernel<2, PAGE16>
                      : rows <= 48 ? attend_kernel<3, PAGE16>
                                   : attend_kernel<4, PAGE16>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, C, Q);
}

template <bool PAGE16>
static void launch_mass(const CacheView &C, const Queries &Q, unsigned blocks, hipStream_t st) {
  const auto kernel = Q.tokens * Q.group <= 48 ? attend_mass_kernel<3, PAGE16> : attend_mass_kernel<4, PAGE16>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, C, Q);
}

int attend_workspace(const CacheView &C, const compactor_cache_query_t *query, const AttendKernels &kernels, size_t *bytes) {
  const int rc = query_check(query, C);
  if (rc) return rc;
  if (!bytes) return COMPACTOR_EINVAL;
  *bytes = attend_plan(C, query, kernels).bytes();
  return COMPACTOR_OK;
}

int attend_call(const CacheView &C, const compactor_cache_query_t *query, const AttendKernels &kernels, bool row16, void *workspace,
                size_t workspace_bytes, void *stream) {
  const int rc = query_check(query, C);
  if (rc) return rc;
  if (!query->q || !query->out || query->out == query->q) return COMPACTOR_EINVAL;
  if (query->q_stride_b < 0 || query->q_stride_l < 0 || query->q_stride_t < 0 || query->q_stride_h < 0 ||
      query->out_stride_b < 0 || query->out_stride_l < 0 || query->out_stride_t < 0 || query->out_stride_h < 0)
    return COMPACTOR_EINVAL;
  if (((reinterpret_cast<uintptr_t>(query->q) | reinterpret_cast<uintptr_t>(query->out)) & 15u) ||
      ((query->q_stride_b | query->q_stride_l | query->q_stride_t | query->q_stride_h | query->out_stride_b |
        query->out_stride_l | query->out_stride_t | query->out_stride_h) & 7) ||
      ((reinterpret_cast<uintptr_t>(query->lse) | reinterpret_cast<uintptr_t>(query->new_tokens)) & 3u))
    return COMPACTOR_EALIGN;
  const AttendPlan A = attend_plan(C, query, kernels);
  const size_t need = A.bytes();
  if (need > 0 && (!workspace || workspace_bytes < need)) return COMPACTOR_EWORKSPACE;
  if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return COMPACTOR_EALIGN;
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  const long long blocks = A.frags_most > 0 ? A.frags_most : heads;
  const bool waves = kernels.bits4 && heads * A.rows >= JOIN_WAVES;
  const long long join = A.joined ? (waves ? (heads * A.rows + 3) / 4 : heads * A.rows) + (query->accumulate && !A.again ? A.frags_most : 0) : 0;
  if (!launchable(blocks, 256) || !launchable(join, 256)) return COMPACTOR_EINVAL;
  Queries Q;
  Q.q = static_cast<const uint16_t *>(query->q);
  Q.out = static_cast<uint16_t *>(query->out);
  Q.lse = query->lse;
  Q.q_stride_b = query->q_stride_b; Q.q_stride_l = query->q_stride_l;
  Q.q_stride_t = query->q_stride_t; Q.q_stride_h = query->q_stride_h;
  Q.out_stride_b = query->out_stride_b; Q.out_stride_l = query->out_stride_l;
  Q.out_stride_t = query->out_stride_t; Q.out_stride_h = query->out_stride_h;
  Q.new_tokens = query->new_tokens;
  Q.tokens = query->tokens;
  Q.group = query->q_heads / C.kv_heads;
  Q.scale = scale_of(query);
  Q.softcap = query->softcap;
  Q.target = A.target;
  Q.split = A.split;
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  Q.frags = A.frags_most > 0 ? reinterpret_cast<Fragment *>(ws) : nullptr;
  ws += A.frags;
  Q.head_frags = A.joined ? reinterpret_cast<int2 *>(ws) : nullptr;
  Q.partial = reinterpret_cast<float *>(ws += A.head_frags);
  Q.stats = reinterpret_cast<float2 *>(ws += A.partial);
  ws += A.stats;
  Q.logits = query->accumulate && !A.again ? reinterpret_cast<float *>(ws) : nullptr;
  Q.weights = A.again ? reinterpret_cast<float *>(ws) : nullptr;
  Q.most = query_most(C, query);
  Q.pitch = A.pitch;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  kernels.attend(C, Q, row16, (unsigned)blocks, st);
  if (A.joined) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    hipLaunchKernelGGL(waves ? attend_join_kernel<true> : attend_join_kernel<false>, dim3((unsigned)join), dim3(256), 0, st, C, Q);
  }
  if (A.again) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    kernels.mass(C, Q, row16, (unsigned)blocks, st);
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

static const AttendKernels &attend_kernels() {
  static const AttendKernels kernels = {
      [](const CacheView &C, const Queries &Q, bool row16, unsigned blocks, hipStream_t st) {
        row16 ? launch_attend<true>(C, Q, blocks, st) : launch_attend<false>(C, Q, blocks, st);
      },
      [](const CacheView &C, const Queries &Q, bool row16, unsigned blocks, hipStream_t st) {
        row16 ? launch_mass<true>(C, Q, blocks, st) : launch_mass<false>(C, Q, blocks, st);
      },
      false, AGAIN_ROWS, AGAIN_BYTES};
  return kernels;
}

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_cache_attention_workspace_size(const compactor_cache_t *cache, const compactor_cache_query_t *query,
                                             size_t *bytes) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_SIZES, &C);
  return rc ? rc : attend_workspace(C, query, attend_kernels(), bytes);
}

int compactor_cache_attention(const compactor_cache_t *cache, const compactor_cache_query_t *query, void *workspace,
                              size_t workspace_bytes, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, query && query->accumulate ? CACHE_STATE : CACHE_ROWS, &C);
  if (rc) return rc;
  // halves of tiles with one origin, and offsets inside one that fit 32 bits
  return attend_call(C, query, attend_kernels(), C.page_size % 16 == 0 && C.slot_stride <= (1 << 24), workspace, workspace_bytes, stream);
}

#pragma GCC visibility pop
}  // extern "C"
