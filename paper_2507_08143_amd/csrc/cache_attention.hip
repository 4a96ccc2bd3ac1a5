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
// wait in the workspace, 4 bytes a slot and query row.
#include <math.h>

#include <algorithm>

#include "cache.h"

namespace cmp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int ATT_TILE = 32;                 // slots a wave takes at a time
constexpr int ATT_WAVES = 4;
constexpr int ATT_STEP = ATT_TILE * ATT_WAVES;
constexpr int MOST_ROWS = 64;                // query rows of a head: G * T
constexpr int MOST_SPLITS = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Queries {
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  long long q_stride_b, q_stride_l, q_stride_t, q_stride_h;
  long long out_stride_b, out_stride_l, out_stride_t, out_stride_h;
  const int32_t *new_tokens;
  int tokens, group;           // T, and G query heads a kv head; row t * G + g of a head
  float scale, softcap;
  int splits, least;           // workgroups a head, and the fewest slots that one takes (whole steps)
  float *partial;              // splits > 1: [head][split][row][D], relative to 2^m
  float2 *stats;               // [head][split][row]: m (base 2) and the sum of 2^(x - m)
  float *logits;               // accumulate: [head][row][pitch], base 2; else null
  int most, pitch;             // slots that there is room for
};

// Slots of one workgroup of a head that holds `count`: whole steps, so that at most Q.splits of them have any.
__device__ __forceinline__ int slots_of_split(const Queries &Q, int count) {
  const int even = (int)(((unsigned)count + (unsigned)Q.splits - 1) / (unsigned)Q.splits);
  const int c = (int)(((unsigned)even + ATT_STEP - 1) / ATT_STEP * ATT_STEP);
  return c > Q.least ? c : Q.least;
}
__device__ __forceinline__ int splits_with_slots(int count, int chunk) {
  return count > 0 ? (int)(((unsigned)count + (unsigned)chunk - 1) / (unsigned)chunk) : 1;
}

// What query row t of n new tokens sees of `count` slots.
__device__ __forceinline__ int sees(int count, int n, int t) { return t < n ? max(count - (n - 1 - t), 0) : 0; }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Over the lanes that share l & 15: swapping halves (quarters) of two copies leaves a lane its own value and that of the
// lane 32 (16) away.
__device__ __forceinline__ float quarters_max(float x) {
  u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quarters_sum(float x) {
  u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 t;
  t[0] = (__bf16)a;
  t[1] = (__bf16)b;
  unsigned u;
  __builtin_memcpy(&u, &t, 4);
  return u;
}

__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

union Piece {
  uint4 u;
  unsigned w[4];
  bf16x8 v;
};

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
  // PAGE16: halves of the tiles at first, first + ATT_STEP, ...
  const long long slot = (long long)first + (lane >> 1) * ATT_STEP + 16 * (lane & 1);
  bool ok = slot < count;
  const int i = page_number(ok ? (unsigned)slot : 0u, C.div_mul, C.div_shift);
  const int page = ok ? p.table[i] : 0;
  ok = ok && page_there(C, page);
  P.off = ok ? page * C.page_stride + ((int)slot - i * C.page_size) * C.slot_stride : 0;
  P.there = __ballot(ok);
}
template <bool PAGE16>
__device__ __forceinline__ void places_fetch(const CacheView &C, const HeadPlace &p, long long first, int count, int lane, Places<PAGE16> &P) {
  const long long slot = first + (lane & 31);
  P.in = slot < count;
  const int i = page_number(P.in ? (unsigned)slot : 0u, C.div_mul, C.div_shift);
  P.page = P.in ? p.table[i] : 0;
  P.at = (int)slot - i * C.page_size;
}
template <bool PAGE16>
__device__ __forceinline__ void places_take(const CacheView &C, Places<PAGE16> &P) {
  const bool ok = P.in && page_there(C, P.page);
  P.off = ok ? P.page * C.page_stride + P.at * C.slot_stride : 0;
  P.there = __ballot(ok);
}

__device__ __forceinline__ long long from_lane(long long x, int lane) {       // the same lane for all
  const unsigned lo = __builtin_amdgcn_readlane((unsigned)x, lane), hi = __builtin_amdgcn_readlane((unsigned)((unsigned long long)x >> 32), lane);
  return (long long)((unsigned long long)hi << 32 | lo);
}

// K or V rows of a tile.  K: pieces 4 kk + (l >> 4) of rows l & 15 of both halves.  V: piece l & 15 of rows 4 (l >> 4) + i of both.
// lane_at (PAGE16): the lane's place in a half, bytes; stride: of a slot, bytes.
template <bool PAGE16, bool K>
__device__ __forceinline__ void load_rows(const uint16_t *base, const Places<PAGE16> &P, int tile, int lane, unsigned lane_at, unsigned stride, Piece (&x)[8]) {
  if (PAGE16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const char *half = reinterpret_cast<const char *>(base + from_lane(P.off, 2 * tile + (i >> 2)));
      x[i].u = load_stream16((K ? half + 64 * (i & 3) : half + (i & 3) * (long long)stride) + lane_at);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long long off = __shfl(P.off, 16 * (i >> 2) + (K ? lane & 15 : 4 * (lane >> 4) + (i & 3)));
      x[i].u = load_stream16(base + off + (K ? 8 * (lane >> 4) + 32 * (i & 3) : 8 * (lane & 15)));
    }
  }
}

// Row r of a head: out = o / sum, lse = ln 2 (m + log2 sum); sum 0: nothing was seen.
__device__ __forceinline__ void finish_row(const CacheView &C, const Queries &Q, const HeadOf &w, int r, int ch, const f32x4 (&o)[2],
                                           float m, float sum) {
  const int t = r / Q.group, qh = w.h * Q.group + r - t * Q.group;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint4 x;
  x.x = pack_bf16(o[0][0] * inv, o[0][1] * inv);
  x.y = pack_bf16(o[0][2] * inv, o[0][3] * inv);
  x.z = pack_bf16(o[1][0] * inv, o[1][1] * inv);
  x.w = pack_bf16(o[1][2] * inv, o[1][3] * inv);
  *reinterpret_cast<uint4 *>(Q.out + w.b * Q.out_stride_b + w.l * Q.out_stride_l + t * Q.out_stride_t + qh * Q.out_stride_h + ch) = x;
  if (ch == 0 && Q.lse != nullptr)
    Q.lse[(((long long)w.b * C.layers + w.l) * Q.tokens + t) * (C.kv_heads * Q.group) + qh] =
        sum == 0.f ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(sum));
}

// Adds the weights of slots [from, to) to the head's mass: 1/G sum over rows of 2^(x - lse2), lse2 = inf for a row without
// weights.
__device__ __forceinline__ void add_mass(const CacheView &C, const Queries &Q, const HeadPlace &hp, const float *lse2, const float *logits,
                                         int R, int from, int to, bool any) {
  if (!any) return;
  const float inv = 1.f / (float)Q.group;
  for (int s = from + (int)threadIdx.x; s < to; s += 256) {
    const SlotPlace at = slot_place(C, hp, s);
    float x = 0.f;
    for (int r = 0; r < R; ++r) x += lse2[r] == INFINITY ? 0.f : exp2_(logits[(long long)r * Q.pitch + s] - lse2[r]);
    if (page_there(C, at.page)) C.mass[state_at(C, hp, at)] += x * inv;
  }
}

template <int NT>
struct AttendLds {
  float o[ATT_WAVES][16][D + 4];
  float m[ATT_WAVES][16 * NT], l[ATT_WAVES][16 * NT];
  float lse2[16 * NT];
};

template <int NT, bool PAGE16>
__global__ __launch_bounds__(256, NT == 1 ? 3 : NT == 2 ? 2 : 1) void attend_kernel(const CacheView C, const Queries Q) {
  __shared__ AttendLds<NT> L;
  const unsigned heads = (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads;
  const unsigned part = blockIdx.x / heads, g = blockIdx.x - part * heads;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, j = lane >> 4;
  const HeadOf w = head_of(C, g);
  const HeadPlace hp = head_place(C, w);
  const int count = held(C, w.b, w.l, w.h), n = tokens_new(Q.new_tokens, w.b, Q.tokens);
  const int R = Q.tokens * Q.group;
  const int chunk = slots_of_split(Q, count);
  const long long begin = (long long)part * chunk;
  if (part > 0 && begin >= count) return;
  const int end = n > 0 ? (int)min(begin + chunk, (long long)count) : 0;        // no queries: no tiles
  const int first = (int)begin + wave * ATT_TILE;                               // of the wave's tiles, ATT_STEP apart
  const int tiles = first < end ? (end - first + ATT_STEP - 1) / ATT_STEP : 0;
  const int seen_by_all = count - (n - 1);
  const uint16_t *kp = C.k + hp.rows, *vp = C.v + hp.rows;

  Places<PAGE16> P;
  if (PAGE16) {
    places_run(C, hp, first, count, lane, P);
  } else {
    places_fetch(C, hp, first, count, lane, P);
    places_take(C, P);
    places_fetch(C, hp, (long long)first + ATT_STEP, count, lane, P);
  }
  // query rows as B operands: lane l has row l & 15, channels 32 kk + 8 (l >> 4) ..
  Piece q[NT][4];
  int see[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 16 * nt + n16, t = r / Q.group;
    see[nt] = r < R ? sees(count, n, t) : 0;
    const uint16_t *qp = Q.q + w.b * Q.q_stride_b + w.l * Q.q_stride_l + t * Q.q_stride_t + (w.h * Q.group + r - t * Q.group) * Q.q_stride_h;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      q[nt][kk].u = make_uint4(0, 0, 0, 0);
      if (see[nt] > 0) q[nt][kk].u = *reinterpret_cast<const uint4 *>(qp + 32 * kk + 8 * j);
    }
  }
  Piece k[8], v[8];
  const unsigned stride = PAGE16 ? 2u * (unsigned)C.slot_stride : 0u, k_at = n16 * stride + 16 * j, v_at = 4 * j * stride + 16 * n16;
  unsigned there = 0;            // bit i: slot i of the tile holds a token whose page is there
  auto tile_there = [&](int tile) {
    if (!PAGE16) return (unsigned)P.there;
    const unsigned two = (unsigned)(P.there >> (2 * (tile & 31)));
    return (two & 1u ? 0xffffu : 0u) | (two & 2u ? 0xffff0000u : 0u);
  };
  if (tiles > 0) {
    load_rows<PAGE16, true>(kp, P, 0, lane, k_at, stride, k);
    load_rows<PAGE16, false>(vp, P, 0, lane, v_at, stride, v);
    there = tile_there(0);
  }

  f32x4 acc[NT][8];
  float m[NT], l[NT];            // of query l & 15: reference of its exponents, the lane's part of their sum
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    l[nt] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[nt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool capped = Q.softcap > 0.f;
  const float to_base2 = Q.scale * LOG2E, to_tanh = capped ? 2.f * LOG2E * Q.scale / Q.softcap : 0.f, cap2 = Q.softcap * LOG2E;
  const bool store = Q.logits != nullptr && count <= Q.most;
  float *logits = Q.logits + (long long)g * R * Q.pitch;

  for (int tile = 0; tile < tiles; ++tile) {
    const int s0 = first + tile * ATT_STEP;
    const bool more = tile + 1 < tiles;
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
    // K of the next tile leaves as soon as its registers are free, V after the second product
    unsigned there_next = 0;
    if (more) {
      if (PAGE16) {
        if (((tile + 1) & 31) == 0) places_run(C, hp, s0 + ATT_STEP, count, lane, P);
      } else {
        places_take(C, P);
        places_fetch(C, hp, (long long)s0 + 2 * ATT_STEP, count, lane, P);
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
    Piece hi[NT], lo[NT];          // P as two bf16 planes, B operands: 16 mantissa bits
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
      if (capped) {                // tanh(y) = 1 - 2 / (e^2y + 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = cap2 - 2.f * cap2 * __builtin_amdgcn_rcpf(exp2_(s[nt][i >> 2][i & 3] * to_tanh) + 1.f);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[nt][i >> 2][i & 3] * to_base2;
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
        float *to = logits + (long long)(16 * nt + n16) * Q.pitch + s0 + 4 * j;
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
      for (int i = 0; i < 4; ++i) {
        hi[nt].w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        lo[nt].w[i] = pack_bf16(x[2 * i] - __uint_as_float(hi[nt].w[i] << 16), x[2 * i + 1] - __uint_as_float(hi[nt].w[i] & 0xffff0000u));
      }
      if (__builtin_expect(ahead, 0)) {
        float *mine = L.o[wave][n16];        // (of the wave alone until the waves meet)
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
    // channels 2 d and 2 d + 1 of the lane's piece, 8 slots each
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      Piece a;
#pragma unroll
      for (int i = 0; i < 4; ++i) a.w[i] = __builtin_amdgcn_perm(v[2 * i + 1].w[c >> 1], v[2 * i].w[c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        acc[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, hi[nt].v, acc[nt][c], 0, 0, 0);
        acc[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, lo[nt].v, acc[nt][c], 0, 0, 0);
      }
    }
    if (more) load_rows<PAGE16, false>(vp, P, (tile + 1) & 31, lane, v_at, stride, v);
    there = there_next;
    __builtin_amdgcn_sched_barrier(0);
  }

  // the four waves meet
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] = quarters_sum(l[nt]);
    if (see[nt] <= 0) {
      m[nt] = -INFINITY;
      l[nt] = 0.f;
    }
    if (j == 0) {
      L.m[wave][16 * nt + n16] = m[nt];
      L.l[wave][16 * nt + n16] = l[nt];
    }
  }
  __syncthreads();
  const bool last = Q.splits == 1;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 16 * nt + n16;
    float top = L.m[0][r];
#pragma unroll
    for (int i = 1; i < ATT_WAVES; ++i) top = fmaxf(top, L.m[i][r]);
    const float f = top == -INFINITY ? 0.f : exp2_(m[nt] - top);
    if (nt > 0) __syncthreads();                    // the last tile of rows has been read
#pragma unroll
    for (int vv = 0; vv < 4; ++vv)
#pragma unroll
      for (int c = 0; c < 8; c += 4)
        *reinterpret_cast<f32x4 *>(&L.o[wave][n16][32 * j + 8 * vv + c]) =
            see[nt] > 0 ? f32x4{acc[nt][c][vv], acc[nt][c + 1][vv], acc[nt][c + 2][vv], acc[nt][c + 3][vv]} * f : f32x4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    // 16 threads a row, 8 channels each
    const int row = 16 * nt + (tid >> 4), ch = 8 * (tid & 15);
    float mm = L.m[0][row], sum = 0.f;
#pragma unroll
    for (int i = 1; i < ATT_WAVES; ++i) mm = fmaxf(mm, L.m[i][row]);
#pragma unroll
    for (int i = 0; i < ATT_WAVES; ++i) sum += mm == -INFINITY ? 0.f : L.l[i][row] * exp2_(L.m[i][row] - mm);
    f32x4 o[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      o[c] = *reinterpret_cast<const f32x4 *>(&L.o[0][tid >> 4][ch + 4 * c]);
#pragma unroll
      for (int i = 1; i < ATT_WAVES; ++i) o[c] += *reinterpret_cast<const f32x4 *>(&L.o[i][tid >> 4][ch + 4 * c]);
    }
    if (row < R) {
      if (last) {
        finish_row(C, Q, w, row, ch, o, mm, sum);
        if (ch == 0) L.lse2[row] = sum == 0.f ? INFINITY : mm + __builtin_amdgcn_logf(sum);
      } else {
        const long long at = ((long long)g * Q.splits + part) * R + row;
        f32x4 *to = reinterpret_cast<f32x4 *>(Q.partial + at * D + ch);
        to[0] = o[0];
        to[1] = o[1];
        if (ch == 0) Q.stats[at] = make_float2(mm, sum);
      }
    }
  }
  if (last && store) {
    __threadfence_block();
    __syncthreads();                                // the workgroup's logits and sums
    add_mass(C, Q, hp, L.lse2, logits, R, 0, count, n > 0);
  }
}

// Second launch: the workgroups of a head meet.  The first R workgroups of a head take a query row each, 16 splits side by side
// and 8 channels a thread; the others add the weights of JOIN_SLOTS slots to the mass.
constexpr int JOIN_SLOTS = 2048;

// Row r's maximum and sum over the splits, by all threads; every thread gets them.
__device__ __forceinline__ float2 join_stats(const float2 *stats, int splits, float (&red)[2][4]) {
  float m = -INFINITY, l = 0.f;
  if ((int)threadIdx.x < splits) {
    const float2 x = stats[0];
    m = x.x;
    l = x.y;
  }
  float top = m;
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  float sum = top == -INFINITY ? 0.f : l * exp2_(m - top);
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if ((threadIdx.x & 63) == 0) red[1][threadIdx.x >> 6] = sum;
  __syncthreads();
  return make_float2(top, (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]));
}

__global__ __launch_bounds__(256) void attend_join_kernel(const CacheView C, const Queries Q, unsigned per_head) {
  __shared__ float red[2][4], part_o[16][D + 4], lse2[MOST_ROWS];
  const unsigned g = blockIdx.x / per_head;
  const int i = (int)(blockIdx.x - g * per_head), tid = threadIdx.x, R = Q.tokens * Q.group;
  const HeadOf w = head_of(C, g);
  const int count = held(C, w.b, w.l, w.h);
  const int splits = splits_with_slots(count, slots_of_split(Q, count));       // at most MOST_SPLITS = the threads
  const long long base = (long long)g * Q.splits * R;
  if (i < R) {
    const float2 all = join_stats(Q.stats + base + (long long)min(tid, splits - 1) * R + i, splits, red);
    const int sl = tid >> 4, ch = 8 * (tid & 15);
    f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    for (int s = sl; s < splits; s += 16) {
      const long long at = base + (long long)s * R + i;
      const float m = Q.stats[at].x, f = all.x == -INFINITY ? 0.f : exp2_(m - all.x);
      const f32x4 *x = reinterpret_cast<const f32x4 *>(Q.partial + at * D + ch);
      o[0] += x[0] * f;
      o[1] += x[1] * f;
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
      finish_row(C, Q, w, i, ch, o, all.x, all.y);
    }
    return;
  }
  const int from = (i - R) * JOIN_SLOTS;
  if (from >= count || count > Q.most) return;
  // every wave takes rows in turn
  for (int r = tid >> 6; r < R; r += 4) {
    float m = -INFINITY, l = 0.f;
    for (int s = tid & 63; s < splits; s += 64) {
      const float2 x = Q.stats[base + (long long)s * R + r];
      const float to = fmaxf(m, x.x);
      l = to == -INFINITY ? 0.f : l * exp2_(m - to) + x.y * exp2_(x.x - to);
      m = to;
    }
    float top = m;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    float sum = top == -INFINITY ? 0.f : l * exp2_(m - top);
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) lse2[r] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
  }
  __syncthreads();
  const int to = count - from < JOIN_SLOTS ? count : from + JOIN_SLOTS;
  add_mass(C, Q, head_place(C, w), lse2, Q.logits + (long long)g * R * Q.pitch, R, from, to, tokens_new(Q.new_tokens, w.b, Q.tokens) > 0);
}

static int query_check(const compactor_cache_query_t *q, const CacheView &C) {
  if (!q) return COMPACTOR_EINVAL;
  if (q->tokens < 1 || q->q_heads < C.kv_heads || q->q_heads % C.kv_heads || q->max_tokens < 0) return COMPACTOR_EINVAL;
  if ((long long)(q->q_heads / C.kv_heads) * q->tokens > 64) return COMPACTOR_EUNSUPPORTED;
  if (!(q->scale >= 0.f) || !isfinite(q->scale) || !(q->softcap >= 0.f) || !isfinite(q->softcap)) return COMPACTOR_EINVAL;
  return COMPACTOR_OK;
}

static int query_most(const CacheView &C, const compactor_cache_query_t *q) {
  return q->max_tokens > 0 && q->max_tokens < C.capacity ? q->max_tokens : C.capacity;
}

struct AttendPlan {
  int rows, splits, least, pitch;
  size_t partial, stats, logits;       // bytes, in this order in the workspace
  size_t bytes() const { return partial + stats + logits; }
};

static AttendPlan attend_plan(const CacheView &C, const compactor_cache_query_t *q) {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    cus = 256;
  AttendPlan A;
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads, most = query_most(C, q);
  A.rows = q->tokens * (q->q_heads / C.kv_heads);
  A.least = 64 * A.rows < 256 ? 256 : (64 * A.rows + ATT_STEP - 1) / ATT_STEP * ATT_STEP;
  long long splits = 24ll * cus / heads;
  splits = std::min(splits, (most + A.least - 1) / A.least);
  A.splits = (int)std::min(std::max(splits, 1ll), (long long)MOST_SPLITS);
  A.pitch = (int)((most + ATT_TILE - 1) / ATT_TILE * ATT_TILE);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  A.partial = A.splits > 1 ? up((size_t)heads * A.splits * A.rows * D * sizeof(float)) : 0;
  A.stats = A.splits > 1 ? up((size_t)heads * A.splits * A.rows * sizeof(float2)) : 0;
  A.logits = q->accumulate ? up((size_t)heads * A.rows * A.pitch * sizeof(float)) : 0;
  return A;
}

template <bool PAGE16>
static void launch_attend(const CacheView &C, const Queries &Q, unsigned blocks, hipStream_t st) {
  const int rows = Q.tokens * Q.group;
  const auto kernel = rows <= 16 ? attend_kernel<1, PAGE16> : rows <= 32 ? attend_kernel<2, PAGE16> : attend_kernel<4, PAGE16>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, C, Q);
}

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_cache_attention_workspace_size(const compactor_cache_t *cache, const compactor_cache_query_t *query,
                                             size_t *bytes) {
  CacheView C;
  int rc = cache_view(cache, CACHE_SIZES, &C);
  if (rc) return rc;
  rc = query_check(query, C);
  if (rc) return rc;
  if (!bytes) return COMPACTOR_EINVAL;
  *bytes = attend_plan(C, query).bytes();
  return COMPACTOR_OK;
}

int compactor_cache_attention(const compactor_cache_t *cache, const compactor_cache_query_t *query, void *workspace,
                              size_t workspace_bytes, void *stream) {
  CacheView C;
  int rc = cache_view(cache, query && query->accumulate ? CACHE_STATE : CACHE_ROWS, &C);
  if (rc) return rc;
  rc = query_check(query, C);
  if (rc) return rc;
  if (!query->q || !query->out) return COMPACTOR_EINVAL;
  if (query->q_stride_b < 0 || query->q_stride_l < 0 || query->q_stride_t < 0 || query->q_stride_h < 0 ||
      query->out_stride_b < 0 || query->out_stride_l < 0 || query->out_stride_t < 0 || query->out_stride_h < 0)
    return COMPACTOR_EINVAL;
  if (((reinterpret_cast<uintptr_t>(query->q) | reinterpret_cast<uintptr_t>(query->out)) & 15u) ||
      ((query->q_stride_b | query->q_stride_l | query->q_stride_t | query->q_stride_h | query->out_stride_b |
        query->out_stride_l | query->out_stride_t | query->out_stride_h) & 7) ||
      ((reinterpret_cast<uintptr_t>(query->lse) | reinterpret_cast<uintptr_t>(query->new_tokens)) & 3u))
    return COMPACTOR_EALIGN;
  const AttendPlan A = attend_plan(C, query);
  const size_t need = A.bytes();
  if (need > 0 && (!workspace || workspace_bytes < need)) return COMPACTOR_EWORKSPACE;
  if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return COMPACTOR_EALIGN;
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  const long long parts = (long long)A.rows + (query->accumulate ? (query_most(C, query) + JOIN_SLOTS - 1) / JOIN_SLOTS : 0);
  if (heads * A.splits > 0x7fffffffll || (A.splits > 1 && heads * parts > 0x7fffffffll)) return COMPACTOR_EINVAL;
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
  Q.scale = query->scale > 0.f ? query->scale : 1.0f / sqrtf((float)D);
  Q.softcap = query->softcap;
  Q.splits = A.splits;
  Q.least = A.least;
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  Q.partial = reinterpret_cast<float *>(ws);
  Q.stats = reinterpret_cast<float2 *>(ws + A.partial);
  Q.logits = query->accumulate ? reinterpret_cast<float *>(ws + A.partial + A.stats) : nullptr;
  Q.most = query_most(C, query);
  Q.pitch = A.pitch;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  // halves of tiles with one origin, and offsets inside one that fit 32 bits
  if (C.page_size % 16 == 0 && C.slot_stride <= (1 << 24))
    launch_attend<true>(C, Q, (unsigned)(heads * A.splits), st);
  else
    launch_attend<false>(C, Q, (unsigned)(heads * A.splits), st);
  if (A.splits > 1) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    hipLaunchKernelGGL(attend_join_kernel, dim3((unsigned)(heads * parts)), dim3(256), 0, st, C, Q, (unsigned)parts);
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
