// Attention of new tokens to a paged cache in 4 bits (see compactor_mx_attention).
//
// As in cache_attention.hip a wave takes tiles of 32 slots and both products take the rows as they arrive in registers.  A slot is 136
// bytes instead of 512, so the numbers' way from 4 bits to bf16 is what comes close to the loads: gfx950 decodes two with their scale in one instruction, 64
// of them a lane and tile, beside some 200 other vector instructions.  Tried and left: the product of K in 4 bits as they are, with queries as sums of three
// numbers of 8 bits (its conversion takes 1 us of every workgroup: 96 heads of 100 slots 7.2 us instead of 6.0, and no long one is faster); rows by way of LDS with two tiles
// on their way (384 heads of 8192 to 32000: 212 us instead of 210, 96 of 2000 17.4 and 16.4); equal shares of all heads' steps for as many workgroups as
// run at a time, whatever heads they are of (1 of 100 slots 8.7 instead of 6.0, 384 of 16000 182 and 176).
//
// K: a lane holds 16 bytes of row l & 15 of each half, channels 32 (l >> 4) .. + 32, one scale; word kk decoded is the A operand of channels
// 32 (l >> 4) + 8 kk .., and the queries are in the same order.  V: word l & 15 (8 channels) of rows 4 (l >> 4) + i of both
// halves; a byte of each of the 8 words, decoded, has channels 2 d and 2 d + 1 of the 8 slots, and 8 byte permutations make the A
// operands of both.
#include <type_traits>

#include "attend.h"
#include "fp4.h"

namespace cmp {

// Where the rows of a wave's tiles lie.  PAGE16: pages hold whole halves of tiles; lane i keeps the origin of half i & 1 of tile i >> 1 of a run of
// 32.  Else lane i keeps that of slot i & 31 of a tile, the page of the one after on its way, and the lanes find each other's in LDS.
template <bool PAGE16>
struct Places4 {
  long long row, state;        // elements
  unsigned long long there;    // bit i: what lane i stands for holds a token
  int page, at;                // !PAGE16: the tile after the next
  bool in;
};
struct Origin { long long row, state; };

template <bool PAGE16>
__device__ __forceinline__ void places4_set(const CacheView &C, bool ok, int page, int at, Places4<PAGE16> &P) {
  P.row = ok ? page * C.page_stride + at * C.slot_stride : 0;
  P.state = ok ? page * C.state_page_stride + at : 0;
  P.there = __ballot(ok);
}
template <bool PAGE16>
__device__ __forceinline__ void places4_run(const CacheView &C, const HeadPlace &p, int first, int count, int lane, Places4<PAGE16> &P) {
  const long long slot = (long long)first + 16 * lane;
  const bool in = slot < count;
  const int i = invariant_quotient(in ? (unsigned)slot : 0u, C.div_mul, C.div_shift);
  const int page = in ? p.table[i] : 0;
  places4_set(C, in && page_there(C, page), page, (int)slot - i * C.page_size, P);
}
template <bool PAGE16>
__device__ __forceinline__ void places4_fetch(const CacheView &C, const HeadPlace &p, long long first, int count, int lane, Places4<PAGE16> &P) {
  const long long slot = first + (lane & 31);
  P.in = slot < count;
  const int i = invariant_quotient(P.in ? (unsigned)slot : 0u, C.div_mul, C.div_shift);
  P.page = P.in ? p.table[i] : 0;
  P.at = (int)slot - i * C.page_size;
}
template <bool PAGE16>
__device__ __forceinline__ void places4_take(const CacheView &C, Places4<PAGE16> &P, Origin *origins, int lane) {
  places4_set(C, P.in && page_there(C, P.page), P.page, P.at, P);
  wave_lds_fence();
  if (lane < 32) origins[lane] = Origin{P.row, P.state};
  wave_lds_fence();
}

// Sixteen bytes on a border of four.
struct __attribute__((packed, aligned(4))) Words4 { unsigned w[4]; };

// K of a tile: the lane's 16 bytes of rows l & 15 of both halves, and their scales.
struct KRows { Piece x[2]; unsigned scale[2]; };
template <bool PAGE16>
__device__ __forceinline__ void load_k(const CacheView &C, const HeadPlace &hp, const Places4<PAGE16> &P, const Origin *origins, int tile, int lane,
                                       unsigned lane_at, KRows &k) {
  const int n16 = lane & 15, j = lane >> 4;
  const char *rows = reinterpret_cast<const char *>(C.k + hp.rows);
  const unsigned char *scales = reinterpret_cast<const unsigned char *>(C.k_scales + hp.state);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (PAGE16) {
      k.x[h].u = *reinterpret_cast<const uint4 *>(rows + 2 * from_lane(P.row, 2 * tile + h) + lane_at);
      k.scale[h] = (scales + 4 * from_lane(P.state, 2 * tile + h))[4u * n16 + j];
    } else {
      const Origin o = origins[16 * h + n16];
      k.x[h].u = *reinterpret_cast<const uint4 *>(rows + 2 * o.row + 16 * j);
      k.scale[h] = (scales + 4 * o.state)[j];
    }
  }
}
// V of a tile: word l & 15 of rows 4 (l >> 4) + (i & 3) of half i >> 2, and the four scales of each.
struct VRows { unsigned x[8], scales[8]; };
template <bool PAGE16>
__device__ __forceinline__ void load_v(const CacheView &C, const HeadPlace &hp, const Places4<PAGE16> &P, const Origin *origins, int tile, int lane,
                                       unsigned lane_at, unsigned stride, VRows &v) {
  const int n16 = lane & 15, j = lane >> 4;
  const char *rows = reinterpret_cast<const char *>(C.v + hp.rows);
  const uint32_t *scales = C.v_scales + hp.state;
  if (PAGE16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char *half = rows + 2 * from_lane(P.row, 2 * tile + h);
#pragma unroll
      for (int i = 0; i < 4; ++i) v.x[4 * h + i] = *reinterpret_cast<const unsigned *>(half + i * (long long)stride + lane_at);
      const Words4 s = *reinterpret_cast<const Words4 *>(scales + from_lane(P.state, 2 * tile + h) + 4u * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) v.scales[4 * h + i] = s.w[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Origin o = origins[16 * (i >> 2) + 4 * j + (i & 3)];
      v.x[i] = *reinterpret_cast<const unsigned *>(rows + 2 * o.row + 4 * n16);
      v.scales[i] = scales[o.state];
    }
  }
}

// Products of K's rows with the queries: query l & 15, slots 4 (l >> 4) + v of each half.
template <int NT>
__device__ __forceinline__ void product_k(const KRows &k, const Piece (&q)[NT][4], f32x4 (&s)[NT][2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float scale = __uint_as_float(k.scale[h] << 23);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      Piece a;
      a.u = fp4_decode(k.x[h].w[kk], scale);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, q[nt][kk].v, s[nt][h], 0, 0, 0);
    }
  }
}
// A operands of channels 2 d and 2 d + 1 of the lane's words of V.
template <int d>
__device__ __forceinline__ void v_operands(const VRows &v, const float (&scale)[8], Piece (&a)[2]) {
  unsigned p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = fp4_pair<d>(v.x[i], scale[i]);
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) a[c].w[i] = __builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], c ? 0x07060302u : 0x05040100u);
}
// Adds weights (hi + lo) times them.
template <int NT, int d>
__device__ __forceinline__ void product_v(const VRows &v, const float (&scale)[8], const Piece (&hi)[NT], const Piece (&lo)[NT], f32x4 (&acc)[NT][8]) {
  Piece a[2];
  v_operands<d>(v, scale, a);
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      acc[nt][2 * d + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c].v, hi[nt].v, acc[nt][2 * d + c], 0, 0, 0);
      acc[nt][2 * d + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c].v, lo[nt].v, acc[nt][2 * d + c], 0, 0, 0);
    }
}
// Two weights as sums of two bf16 numbers: 2^-17 of them is lost.  (V that is written here holds no infinities, whose product with a lower part of the other sign would be none.)
__device__ __forceinline__ void split4(float x0, float x1, unsigned &hi, unsigned &lo) {
  hi = pack_bf16(x0, x1);
  lo = pack_bf16(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xffff0000u));
}

// Logits of a tile over `unit`, which makes them of base 2 (capped ones are of base 2 as they are: unit_of()).  whole: all of its slots are there and
// seen by every query, else there_at has bit 16 (i >> 2) + (i & 3) for the lane's i-th slot and `upto` says what its query sees of them.
__device__ __forceinline__ float unit_of(const Scaling &scaling) { return scaling.capped ? 1.f : scaling.to_base2; }
template <int N>
__device__ __forceinline__ void cap_logits(const Scaling &scaling, float (&x)[N]) {
  // most logits are in the middle of the cap, where the series does
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(x[i]));
  if (__any(!(top * scaling.to_y < 0.25f))) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = capped_logit(scaling, x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = capped_small(scaling, x[i]);
  }
}
__device__ __forceinline__ void tile_logits(const Scaling &scaling, const f32x4 (&s)[2], bool whole, unsigned there_at, int upto, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = s[i >> 2][i & 3];
  if (scaling.capped) cap_logits(scaling, x);
  if (__builtin_expect(!whole, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = 16 * (i >> 2) + (i & 3);
      x[i] = (there_at >> at & 1u) && at < upto ? x[i] : -INFINITY;
    }
  }
}

template <bool PAGE16>
__device__ __forceinline__ unsigned tile4_there(const Places4<PAGE16> &P, int tile) {
  if (!PAGE16) return (unsigned)P.there;
  const unsigned two = (unsigned)(P.there >> (2 * (tile & 31)));
  return (two & 1u ? 0xffffu : 0u) | (two & 2u ? 0xffff0000u : 0u);
}

template <int NT, bool PAGE16>
struct Attend4Lds {
  float o[ATT_WAVES][16][D + 4];
  Origin origins[ATT_WAVES][PAGE16 ? 1 : 32];
  float m[ATT_WAVES][16 * NT], l[ATT_WAVES][16 * NT];
  float lse2[16 * NT];
  int none;
};

// The row of a later token is no part of an earlier one's output even where it holds no number (0 * NaN).  In a tile that is not `whole`: of rows that
// not all queries see, groups that are NaN are left out of the product, and make NaN of the outputs of those that see them; so are rows that are not there.
template <int NT>
__device__ __forceinline__ void mask_v(const CacheView &C, const HeadPlace &hp, VRows &v, unsigned there, int s0, int left, int seen_by_all, const int (&see)[NT],
                                       f32x4 (&acc)[NT][8]) {
  const int lane = threadIdx.x & 63, n16 = lane & 15, j = lane >> 4;
  const unsigned there_at = there >> (4 * j), group_shift = 8 * (n16 >> 2);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = 16 * (i >> 2) + (i & 3);
    const bool ahead = s0 + 4 * j + at >= seen_by_all && (v.scales[i] >> group_shift & 0xffu) == FP4_NAN;
    const bool keep = there_at >> at & 1u;
    odd |= keep && ahead;
    if (!keep || ahead) v.x[i] = v.scales[i] = 0;
  }
  if (!__any(odd)) return;
#pragma unroll 1
  for (int i = max(seen_by_all - s0, 0); i < min(left, ATT_TILE); ++i) {
    if (!(there >> i & 1u)) continue;
    const unsigned scales = C.v_scales[state_at(C, hp, slot_place(C, hp, s0 + i))];
    const bool poison = (scales >> (8 * j) & 0xffu) == FP4_NAN;      // the lane's sums are those of group l >> 4
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (poison && s0 + i < see[nt])
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[nt][c] = f32x4{NAN, NAN, NAN, NAN};
  }
}
__device__ __forceinline__ void v_scale_of(const VRows &v, float (&scale)[8]) {
  const unsigned group_shift = 8 * ((threadIdx.x & 15) >> 2);
#pragma unroll
  for (int i = 0; i < 8; ++i) scale[i] = __uint_as_float((v.scales[i] >> group_shift & 0xffu) << 23);
}

// The workgroup's part of a head; false: there is none.
__device__ __forceinline__ bool part_of(const CacheView &C, const Queries &Q, Fragment &part, int &fragment) {
  fragment = (int)blockIdx.x;
  if (!(Q.target > 0 ? scan_part<true>(C, Q, fragment, part) : split_part<true>(C, Q, part, fragment))) {
    if (threadIdx.x == 0) Q.frags[fragment].head = -1;
    return false;
  }
  if (Q.frags != nullptr && threadIdx.x == 0) {
    Q.frags[fragment] = part;
    if (Q.head_frags != nullptr && part.step0 == 0) Q.head_frags[part.head] = make_int2(part.first, part.parts);
  }
  return true;
}

// Workgroups a unit: three of up to 16 rows (with four, 128 registers, 384 heads of 8192 to 32000, 4 rows: 242 us instead of 210), one of more than 48 (two of
// 256 registers: 192 heads of 16000 to 32000, 64 rows, 939 us instead of 424; of 40 rows, 330 with two and 500 with one).
template <int NT, bool PAGE16>
__global__ __launch_bounds__(256, NT == 1 ? 3 : NT <= 3 ? 2 : 1) void attend4_kernel(const CacheView C, const Queries Q) {
  __shared__ Attend4Lds<NT, PAGE16> L;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, j = lane >> 4;
  const int R = Q.tokens * Q.group;
  Fragment part;
  int fragment;
  if (!part_of(C, Q, part, fragment)) return;
  const HeadOf w = head_of(C, (unsigned)part.head);
  const HeadPlace hp = head_place(C, w);
  const int count = part.count, n = part.n;
  if (tid == 0) L.none = 0;
  const Run run = run_of(part, wave);
  const int first = run.first, tiles = run.tiles;
  const int seen_by_all = count - (n - 1);
  Origin *origins = L.origins[wave];

  Places4<PAGE16> P;
  if (PAGE16) {
    places4_run(C, hp, first, count, lane, P);
  } else {
    places4_fetch(C, hp, first, count, lane, P);
    places4_take(C, P, origins, lane);
    places4_fetch(C, hp, (long long)first + ATT_TILE, count, lane, P);
  }
  Piece q[NT][4];
  int see[NT];
  load_queries<NT, true>(Q, w, R, count, n, q, see);
  KRows k;
  VRows v;
  const unsigned stride = PAGE16 ? 2u * (unsigned)C.slot_stride : 0u, k_at = n16 * stride + 16 * j, v_at = 4 * j * stride + 4 * n16;
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
  const float unit = unit_of(scaling);
  const bool store = Q.logits != nullptr && count <= Q.most;
  float *logits = Q.logits + (long long)part.head * R * Q.pitch;

  unsigned there = 0;            // bit i: slot i of the tile holds a token whose page is there
  auto one_tile = [&](int tile, auto another) {
    constexpr bool more = decltype(another)::value;
    const int s0 = first + tile * ATT_TILE;
    f32x4 s[NT][2];
    product_k<NT>(k, q, s);
    // V of this tile has the places still: where lanes find them in LDS, they are loaded again before the next tile's come
    const int left = count - s0;
    if (left < 32) there &= (1u << left) - 1u;              // left >= 1
    const bool whole = there == 0xffffffffu && s0 + ATT_TILE <= seen_by_all;      // the same for all lanes
    const unsigned there_at = there >> (4 * j);             // bit 16 (i >> 2) + (i & 3): the lane's i-th slot
    unsigned there_next = 0;
    if constexpr (more) {
      if (PAGE16) {
        if (((tile + 1) & 31) == 0) places4_run(C, hp, s0 + ATT_TILE, count, lane, P);
      } else {
        places4_take(C, P, origins, lane);
        places4_fetch(C, hp, (long long)s0 + 2 * ATT_TILE, count, lane, P);
      }
      load_k<PAGE16>(C, hp, P, origins, (tile + 1) & 31, lane, k_at, k);
      there_next = tile4_there(P, tile + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (__builtin_expect(!whole, 0)) mask_v<NT>(C, hp, v, there, s0, left, seen_by_all, see, acc);
    Piece hi[NT], lo[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
      tile_logits(scaling, s[nt], whole, there_at, see[nt] - s0 - 4 * j, x);
      if (store && 16 * nt + n16 < R) {
        float *to = logits + (long long)(16 * nt + n16) * Q.pitch + s0 + 4 * j;
        *reinterpret_cast<f32x4 *>(to) = f32x4{x[0], x[1], x[2], x[3]} * unit;
        *reinterpret_cast<f32x4 *>(to + 16) = f32x4{x[4], x[5], x[6], x[7]} * unit;
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
      // the reference moves only when it has fallen 2^8 behind: weights up to 2^8 keep their precision
      if (__any(top * unit > m[nt] + 8.f)) {
        const float to = fmaxf(m[nt], quarters_max(top) * unit), f = to == -INFINITY ? 1.f : exp2_(m[nt] - to);
        m[nt] = to;
        l[nt] *= f;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[nt][c] *= f;
      }
      const float ref = m[nt] == -INFINITY ? 0.f : m[nt];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = exp2_(fmaf(x[i], unit, -ref));
        sum += x[i];
      }
      l[nt] += sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) split4(x[2 * i], x[2 * i + 1], hi[nt].w[i], lo[nt].w[i]);
    }
    float scale[8];
    v_scale_of(v, scale);
    product_v<NT, 0>(v, scale, hi, lo, acc);
    product_v<NT, 1>(v, scale, hi, lo, acc);
    product_v<NT, 2>(v, scale, hi, lo, acc);
    product_v<NT, 3>(v, scale, hi, lo, acc);
    if constexpr (more) load_v<PAGE16>(C, hp, P, origins, (tile + 1) & 31, lane, v_at, stride, v);
    there = there_next;
    __builtin_amdgcn_sched_barrier(0);
  };
  // No load of rows of the loop is under a condition, or the compiler would have to wait for V where it waits for K; nor is one
  // issued that nobody wants: the barrier below would wait for it.
  if (tiles > 0) {
    load_k<PAGE16>(C, hp, P, origins, 0, lane, k_at, k);
    load_v<PAGE16>(C, hp, P, origins, 0, lane, v_at, stride, v);
    there = tile4_there(P, 0);
    for (int tile = 0; tile + 1 < tiles; ++tile) one_tile(tile, std::true_type());
    one_tile(tiles - 1, std::false_type());
  }
  waves_meet<NT>(C, Q, w, part, fragment, L, acc, m, l, see);
  if (part.parts == 1 && store && n > 0) mass_here(C, Q, hp, logits, R, count, L.lse2, &L.none);
}

// ------------------------------------------------------------------------------------------ up to eight query rows
// Half of the sixteen columns are then nobody's.  Lanes l & 15 = c and c + 8 share the logits of row c: the first has those of the tile's first half, the
// other those of the second, which leaves half of the way from logits to weights; and in the product with V column c has the upper parts of all weights and c + 8 the
// lower ones, which leaves half of its products.  (us in sixteen columns / so: 384 heads of 8192 to 32000, 8 rows, capped 240 / 223, 4 rows 208 / 210; 96 of 16000, 4 rows, pages
// of 24 51 / 49; 1 of 1000 11.4 / 11.1.)
constexpr int FEW_ROWS = 8;

// x, but in lanes c + 8 of 16 (lower: in lanes c) the y of the lane 8 away.
template <bool lower>
__device__ __forceinline__ unsigned with_other(unsigned x, unsigned y) {
  return (unsigned)__builtin_amdgcn_update_dpp((int)x, (int)y, 0x128, 0xf, lower ? 0x3 : 0xc, false);
}
__device__ __forceinline__ float other_half(float x) {             // that of the lane 8 away
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, false));
}
template <int d>
__device__ __forceinline__ void product_few(const VRows &v, const float (&scale)[8], const Piece &p, f32x4 (&acc)[8]) {
  Piece a[2];
  v_operands<d>(v, scale, a);
#pragma unroll
  for (int c = 0; c < 2; ++c) acc[2 * d + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c].v, p.v, acc[2 * d + c], 0, 0, 0);
}

template <bool PAGE16>
__global__ __launch_bounds__(256, 3) void attend4_few_kernel(const CacheView C, const Queries Q) {
  __shared__ Attend4Lds<1, PAGE16> L;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, j = lane >> 4;
  const int R = Q.tokens * Q.group, half = n16 >> 3, row = n16 & 7;
  Fragment part;
  int fragment;
  if (!part_of(C, Q, part, fragment)) return;
  const HeadOf w = head_of(C, (unsigned)part.head);
  const HeadPlace hp = head_place(C, w);
  const int count = part.count, n = part.n;
  if (tid == 0) L.none = 0;
  const Run run = run_of(part, wave);
  const int first = run.first, tiles = run.tiles;
  const int seen_by_all = count - (n - 1);
  Origin *origins = L.origins[wave];
  Places4<PAGE16> P;
  if (PAGE16) {
    places4_run(C, hp, first, count, lane, P);
  } else {
    places4_fetch(C, hp, first, count, lane, P);
    places4_take(C, P, origins, lane);
    places4_fetch(C, hp, (long long)first + ATT_TILE, count, lane, P);
  }
  Piece q[1][4];
  int see[1];
  load_queries<1, true>(Q, w, R, count, n, q, see);
  see[0] = (int)with_other<false>((unsigned)see[0], (unsigned)see[0]);          // of row l & 7
  KRows k;
  VRows v;
  const unsigned stride = PAGE16 ? 2u * (unsigned)C.slot_stride : 0u, k_at = n16 * stride + 16 * j, v_at = 4 * j * stride + 4 * n16;
  f32x4 acc[1][8];               // columns c and c + 8: sums of the upper and the lower parts
  float m = -INFINITY, l = 0.f;  // of row l & 7: reference of its exponents, the lane's part of their sum
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[0][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const Scaling scaling = scaling_of(Q);
  const float unit = unit_of(scaling);
  const bool store = Q.logits != nullptr && count <= Q.most && row < R;
  float *logits = Q.logits + ((long long)part.head * R + min(row, R - 1)) * Q.pitch + 16 * half + 4 * j;

  unsigned there = 0;            // bit i: slot i of the tile holds a token whose page is there
  auto one_tile = [&](int tile, auto another) {
    constexpr bool more = decltype(another)::value;
    const int s0 = first + tile * ATT_TILE;
    f32x4 s[1][2];
    product_k<1>(k, q, s);
    const int left = count - s0;
    if (left < 32) there &= (1u << left) - 1u;              // left >= 1
    const bool whole = there == 0xffffffffu && s0 + ATT_TILE <= seen_by_all;      // the same for all lanes
    unsigned there_next = 0;
    if constexpr (more) {
      if (PAGE16) {
        if (((tile + 1) & 31) == 0) places4_run(C, hp, s0 + ATT_TILE, count, lane, P);
      } else {
        places4_take(C, P, origins, lane);
        places4_fetch(C, hp, (long long)s0 + 2 * ATT_TILE, count, lane, P);
      }
      load_k<PAGE16>(C, hp, P, origins, (tile + 1) & 31, lane, k_at, k);
      there_next = tile4_there(P, tile + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (__builtin_expect(!whole, 0)) mask_v<1>(C, hp, v, there, s0, left, seen_by_all, see, acc);
    float x[4];                  // slots 16 half + 4 j + i of row l & 7
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(with_other<false>(__float_as_uint(s[0][0][i]), __float_as_uint(s[0][1][i])));
    if (scaling.capped) cap_logits(scaling, x);
    if (__builtin_expect(!whole, 0)) {
      const unsigned there_at = there >> (16 * half + 4 * j);
      const int upto = see[0] - s0 - 16 * half - 4 * j;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (there_at >> i & 1u) && i < upto ? x[i] : -INFINITY;
    }
    if (store) *reinterpret_cast<f32x4 *>(logits + s0) = f32x4{x[0], x[1], x[2], x[3]} * unit;
    float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    // the reference moves only when it has fallen 2^8 behind: weights up to 2^8 keep their precision
    if (__any(top * unit > m + 8.f)) {
      top = quarters_max(top);
      const float to = fmaxf(m, fmaxf(top, other_half(top)) * unit), f = to == -INFINITY ? 1.f : exp2_(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[0][c] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = exp2_(fmaf(x[i], unit, -ref));
    l += (x[0] + x[1]) + (x[2] + x[3]);
    unsigned hi[2], lo[2];
    split4(x[0], x[1], hi[0], lo[0]);
    split4(x[2], x[3], hi[1], lo[1]);
    Piece p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      p.w[i] = with_other<false>(hi[i], lo[i]);
      p.w[2 + i] = with_other<true>(lo[i], hi[i]);
    }
    float scale[8];
    v_scale_of(v, scale);
    product_few<0>(v, scale, p, acc[0]);
    product_few<1>(v, scale, p, acc[0]);
    product_few<2>(v, scale, p, acc[0]);
    product_few<3>(v, scale, p, acc[0]);
    if constexpr (more) load_v<PAGE16>(C, hp, P, origins, (tile + 1) & 31, lane, v_at, stride, v);
    there = there_next;
    __builtin_amdgcn_sched_barrier(0);
  };
  if (tiles > 0) {
    load_k<PAGE16>(C, hp, P, origins, 0, lane, k_at, k);
    load_v<PAGE16>(C, hp, P, origins, 0, lane, v_at, stride, v);
    there = tile4_there(P, 0);
    for (int tile = 0; tile + 1 < tiles; ++tile) one_tile(tile, std::true_type());
    one_tile(tiles - 1, std::false_type());
  }
  l += other_half(l);
#pragma unroll
  for (int c = 0; c < 8; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[0][c][i] += other_half(acc[0][c][i]);
  float ms[1] = {m}, ls[1] = {l};
  if (half) see[0] = 0;            // no row of its own
  waves_meet<1>(C, Q, w, part, fragment, L, acc, ms, ls, see);
  if (part.parts == 1 && Q.logits != nullptr && count <= Q.most && n > 0)
    mass_here(C, Q, hp, Q.logits + (long long)part.head * R * Q.pitch, R, count, L.lse2, &L.none);
}

// Weights of many rows from K, which is read again (third launch): see attend_mass_kernel.
template <int NT, bool PAGE16>
__global__ __launch_bounds__(256) void attend4_mass_kernel(const CacheView C, const Queries Q) {
  __shared__ float2 stats[256];
  __shared__ float lse2[MOST_ROWS];
  __shared__ Origin all_origins[ATT_WAVES][PAGE16 ? 1 : 32];
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
  Origin *origins = all_origins[wave];
  Places4<PAGE16> P;
  if (PAGE16) {
    places4_run(C, hp, first, count, lane, P);
  } else {
    places4_fetch(C, hp, first, count, lane, P);
    places4_take(C, P, origins, lane);
    places4_fetch(C, hp, (long long)first + ATT_TILE, count, lane, P);
  }
  Piece q[NT][4];
  KRows k;
  int see[NT];
  load_queries<NT, true>(Q, w, R, count, part.n, q, see);
  const unsigned k_at = PAGE16 ? n16 * (2u * (unsigned)C.slot_stride) + 16 * j : 0u;
  unsigned there = 0;
  if (tiles > 0) {
    load_k<PAGE16>(C, hp, P, origins, 0, lane, k_at, k);
    there = tile4_there(P, 0);
  }
  row_sums(Q, part, R, stats, lse2, &none);
  __syncthreads();
  float z[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) z[nt] = see[nt] > 0 ? lse2[16 * nt + n16] : INFINITY;
  const Scaling scaling = scaling_of(Q);
  const float unit = unit_of(scaling);
  float *weights = Q.weights + (long long)part.head * Q.pitch;

  auto one_tile = [&](int tile, auto another) {
    constexpr bool more = decltype(another)::value;
    const int s0 = first + tile * ATT_TILE;
    f32x4 s[NT][2];
    product_k<NT>(k, q, s);
    unsigned there_next = 0;
    if constexpr (more) {
      if (PAGE16) {
        if (((tile + 1) & 31) == 0) places4_run(C, hp, s0 + ATT_TILE, count, lane, P);
      } else {
        places4_take(C, P, origins, lane);
        places4_fetch(C, hp, (long long)s0 + 2 * ATT_TILE, count, lane, P);
      }
      load_k<PAGE16>(C, hp, P, origins, (tile + 1) & 31, lane, k_at, k);
      there_next = tile4_there(P, tile + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int left = count - s0;
    if (left < 32) there &= (1u << left) - 1u;
    const bool whole = there == 0xffffffffu && s0 + ATT_TILE <= seen_by_all;
    float sum[8] = {};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
      tile_logits(scaling, s[nt], whole, there >> (4 * j), see[nt] - s0 - 4 * j, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += z[nt] == INFINITY ? 0.f : exp2_(fmaf(x[i], unit, -z[nt]));
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

// Weights from K, read again: 64 bytes a slot against 8 for every row, which pays where the last cache does not hold the logits.  us with K / logits: 192 heads of
// 4000 to 8000, 40 rows (logits of 183 MB) 136 / 173, 2000 to 4000 (46 MB) 67 / 60; 96 of 16000 to 32000, 20 rows (183 MB) 157 / 169, 16 rows (146 MB) 125 / 140; 96 of
// 5000 to 9831, 20 rows (57 MB) 64 / 55; 384 of 8000 to 16000, 10 rows (184 MB) 249 / 242.
constexpr int AGAIN4_ROWS = 12;
constexpr size_t AGAIN4_BYTES = 128u << 20;

template <bool PAGE16>
static void launch_attend4(const CacheView &C, const Queries &Q, unsigned blocks, hipStream_t st) {
  const int rows = Q.tokens * Q.group;
  const auto kernel = rows <= FEW_ROWS ? attend4_few_kernel<PAGE16>
                      : rows <= 16 ? attend4_kernel<1, PAGE16>
                      : rows <= 32 ? attend4_kernel<2, PAGE16>
                      : rows <= 48 ? attend4_kernel<3, PAGE16>
                                   : attend4_kernel<4, PAGE16>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, C, Q);
}
template <bool PAGE16>
static void launch_mass4(const CacheView &C, const Queries &Q, unsigned blocks, hipStream_t st) {
  const int rows = Q.tokens * Q.group;
  const auto kernel = rows <= 16   ? attend4_mass_kernel<1, PAGE16>
                      : rows <= 32 ? attend4_mass_kernel<2, PAGE16>
                      : rows <= 48 ? attend4_mass_kernel<3, PAGE16>
                                   : attend4_mass_kernel<4, PAGE16>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, C, Q);
}

static const AttendKernels &attend4_kernels() {
  static const AttendKernels kernels = {
      [](const CacheView &C, const Queries &Q, bool row16, unsigned blocks, hipStream_t st) {
        row16 ? launch_attend4<true>(C, Q, blocks, st) : launch_attend4<false>(C, Q, blocks, st);
      },
      [](const CacheView &C, const Queries &Q, bool row16, unsigned blocks, hipStream_t st) {
        row16 ? launch_mass4<true>(C, Q, blocks, st) : launch_mass4<false>(C, Q, blocks, st);
      },
      true, AGAIN4_ROWS, AGAIN4_BYTES};
  return kernels;
}

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_mx_attention_workspace_size(const compactor_mx_cache_t *cache, const compactor_cache_query_t *query, size_t *bytes) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_SIZES, &C);
  return rc ? rc : attend_workspace(C, query, attend4_kernels(), bytes);
}

int compactor_mx_attention(const compactor_mx_cache_t *cache, const compactor_cache_query_t *query, void *workspace,
                            size_t workspace_bytes, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, query && query->accumulate ? CACHE_STATE : CACHE_ROWS, &C);
  if (rc) return rc;
  // halves of tiles with one origin, and offsets inside one that fit 32 bits
  return attend_call(C, query, attend4_kernels(), C.page_size % 16 == 0 && C.slot_stride <= (1 << 24), workspace, workspace_bytes, stream);
}

#pragma GCC visibility pop
}  // extern "C"
