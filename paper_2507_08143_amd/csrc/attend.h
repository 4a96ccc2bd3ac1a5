// What the kernels of attention to a paged cache share, whatever its rows are held in: how heads are cut into fragments, how a
// fragment's rows are finished and its weights added to the mass, and how logits come out of products (see compactor_cache_attention).
#pragma once

#include <math.h>

#include <algorithm>

#include "cache.h"
#include "fragments.h"

namespace cmp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int ATT_TILE = 32;                 // slots a wave takes at a time
constexpr int ATT_WAVES = 4;
constexpr int ATT_STEP = ATT_TILE * ATT_WAVES;
constexpr int MOST_ROWS = 64;                // query rows of a head: G * T
constexpr int SPLIT_ALL = 4096, SPLIT_MOST = 8;        // more heads: parts of all of them, and of one, at most
constexpr int ATT_ALONE = 8;                 // steps of a head up to which one workgroup takes all of it
// Weights of more than 32 rows are found from K instead of from logits that are more than the last cache holds: 256 bytes a slot read again, against 4
// written and 4 read for every row.  us with K / logits: 96 heads of 18000, 64 rows 352 / 434, 40 rows 311 / 339, 32 rows 293 / 294, 28 rows 290 / 277, 20 rows
// 283 / 253; 192 such heads, 64 rows 643 / 837, 32 rows 550 / 577, 28 rows 546 / 550, 20 rows 534 / 503; 24 of them, whose logits (110 MB for 64 rows) stay near, 64 rows
// 106 / 110, 40 rows 87 / 87, 32 rows 74 / 69.
constexpr int AGAIN_ROWS = 32;
constexpr size_t AGAIN_BYTES = 256u << 20;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A part of a head that one workgroup does.
struct Fragment {
  int head;                    // -1: there is none
  int count, n;                // tokens that it holds, and queries
  int step0, step1;            // steps of the part
  int first, parts;            // the head's first fragment, and how many it has
};

struct Queries {
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  long long q_stride_b, q_stride_l, q_stride_t, q_stride_h;
  long long out_stride_b, out_stride_l, out_stride_t, out_stride_h;
  const int32_t *new_tokens;
  int tokens, group;           // T, and G query heads a kv head; row t * G + g of a head
  float scale, softcap;
  int target;                  // > 0: whole fragments that there are to be (scan_part)
  int split;                   // else: workgroups a head (split_part)
  Fragment *frags;             // null where nobody asks for them: every workgroup has a whole head, and no third launch follows
  int2 *head_frags;            // [head]: its first fragment, and how many; null: every workgroup has a whole head
  float *partial;              // [fragment][row][D], relative to 2^m
  float2 *stats;               // [fragment][row]: m (base 2) and the sum of 2^(x - m)
  float *logits;               // accumulate: [head][row][pitch], base 2; else null
  float *weights;              // or, summed over the rows, [head][pitch] (attend_mass_kernel)
  int most, pitch;             // slots that there is room for
};

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

__device__ __forceinline__ long long from_lane(long long x, int lane) {       // the same lane for all
  const unsigned lo = __builtin_amdgcn_readlane((unsigned)x, lane), hi = __builtin_amdgcn_readlane((unsigned)((unsigned long long)x >> 32), lane);
  return (long long)((unsigned long long)hi << 32 | lo);
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

// What a row's weights are relative to (base 2), inf for a row that has none.  The weights of a row whose sum is NaN are NaN at every slot that
// it sees and at no other: it counts as a row without weights, and *none becomes the most slots that such a row sees.
__device__ __forceinline__ float weights_from(const Queries &Q, int count, int n, int r, float m, float sum, int *none) {
  if (sum != sum) atomicMax(none, sees(count, n, r / Q.group));
  return sum > 0.f ? m + __builtin_amdgcn_logf(sum) : INFINITY;
}

// Weights of the head's slots s .. s + 3, s a multiple of 4, on the way to their mass: what does not depend on the rows' sums leaves
// early (the mass, and the logits of the first MASS_ROWS rows).
constexpr int MASS_ROWS = 4;
struct MassQuad {
  float *mass[4], old[4];
  bool there[4];
  f32x4 x[MASS_ROWS];
};
__device__ __forceinline__ void mass_fetch(const CacheView &C, const Queries &Q, const HeadPlace &hp, const float *logits, int R, int s, int to, MassQuad &M) {
  SlotPlace at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) at[i] = slot_place(C, hp, min(s + i, to - 1));
#pragma unroll
  for (int r = 0; r < MASS_ROWS; ++r) M.x[r] = *reinterpret_cast<const f32x4 *>(logits + (long long)min(r, R - 1) * Q.pitch + s);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool there = page_there(C, at[i].page);
    M.there[i] = s + i < to && there;
    M.mass[i] = C.mass + state_at(C, hp, SlotPlace{there ? at[i].page : 0, at[i].at});
    M.old[i] = *M.mass[i];
  }
}
// 1/G sum over rows of 2^(x - lse2), lse2 and none: weights_from().
__device__ __forceinline__ void mass_add(const Queries &Q, const float *lse2, int none, const float *logits, int R, int s, const MassQuad &M) {
  const float inv = 1.f / (float)Q.group;
  f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
  auto row = [&](int r, const f32x4 &x) {
    const float z = lse2[r];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += z == INFINITY ? 0.f : exp2_(x[i] - z);
  };
#pragma unroll
  for (int r = 0; r < MASS_ROWS; ++r)
    if (r < R) row(r, M.x[r]);
#pragma unroll 8
  for (int r = MASS_ROWS; r < R; ++r) row(r, *reinterpret_cast<const f32x4 *>(logits + (long long)r * Q.pitch + s));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (M.there[i]) *M.mass[i] = s + i < none ? NAN : fmaf(sum[i], inv, M.old[i]);
}

// Steps of ATT_STEP slots of a head: one at least, so that every head has a workgroup that writes its rows.
__device__ __forceinline__ int steps_of(int count, int n) { return n > 0 && count > ATT_STEP ? (int)(((unsigned)count + ATT_STEP - 1) / ATT_STEP) : 1; }
struct HeadSize { int count, n; };           // tokens held, and queries
__device__ __forceinline__ HeadSize head_size(const CacheView &C, const Queries &Q, unsigned g) {
  const HeadOf w = head_of(C, g);
  return HeadSize{held(C, w.b, w.l, w.h), tokens_new(Q.new_tokens, w.b, Q.tokens)};
}

// How long a head is only the device knows, so up to SCAN_HEADS heads every wave finds its workgroup's part by itself, without a
// barrier: heads are cut into fragments of as many steps each, numbered head after head, at most `target` of them beside
// the last of each head.  A few rounds of workgroups keep the chip busy to the end whatever the lengths (16 requests of 68
// to 55778 slots a head, us with fragments of any size in 1 / 2 / 3 / 4 / 6 rounds 212 / 202 / 201 / 202 / 203; 48 of 8192 to 32000 833 / 694 / 657 /
// 652 / 643; 32 of 500 to 16000 131 / 119 / 116 / 116 / 120; cutting every head into the same number of parts 217 / 645 / -).  Heads of (nearly)
// one length need no rounds where whole rounds of units have equal parts (256 heads of 4000: 84 against 89, 512 183 against 213).
//
// What a workgroup does before its first load of rows counts: under load, 26 us of the first case's 202 for 650 instructions
// more.  A launch that plans the fragments for all costs 9 us and saves less (the cases above 210 / 666 / 123).  From SCAN_HEADS
// heads on each is cut into the same few parts (split_part): 1024 heads of 4000, us with a scan / a plan / parts 407 / 384 / 360, of 250 to 8000
// 249 / 237 / 232, 4096 of 2000 1045 / 786 / 692.  -> false: there is no such fragment.
constexpr int SCAN_GROUP = 4;                // of 64 heads whose sizes are fetched together; the first stays
// BITS4: of rows of 4 bits.  Where heads lie side by side two of their rows share a line of memory, so the parts of both with the same slots go to one XCD, whose
// cache it then comes into once: workgroups go round the eight XCDs, those with the same place among eight of two times eight take two parts in turn, and
// of two neighbours' parts the same of both come one behind the other.  `fragment` becomes the number under which its results are kept.
template <bool BITS4 = false>
__device__ __forceinline__ bool scan_part(const CacheView &C, const Queries &Q, int &fragment, Fragment &F) {
  if (BITS4 && (blockIdx.x | 15u) < gridDim.x) fragment = (fragment & ~15) | (fragment & 7) << 1 | (fragment >> 3 & 1);
  const int heads = C.nreq * C.layers * C.kv_heads, lane = threadIdx.x & 63;
  HeadSize size[SCAN_GROUP];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int i = 0; i < SCAN_GROUP; ++i)
      if (i == 0 || h0 + 64 * i < heads) size[i] = head_size(C, Q, (unsigned)min(h0 + 64 * i + lane, heads - 1));
  };
  auto steps_at = [&](int h0, int i) { return h0 + 64 * i + lane < heads ? steps_of(size[i].count, size[i].n) : 0; };
#pragma unroll
  for (int i = 0; i < SCAN_GROUP; ++i) size[i] = HeadSize{0, 0};
  int mine = 0, longest = 0;
  for (int h0 = (heads - 1) / (64 * SCAN_GROUP) * (64 * SCAN_GROUP); h0 >= 0; h0 -= 64 * SCAN_GROUP) {
    fetch(h0);
#pragma unroll
    for (int i = 0; i < SCAN_GROUP; ++i) {
      mine += steps_at(h0, i);
      longest = max(longest, steps_at(h0, i));
    }
  }
  const int total = __builtin_amdgcn_readlane(wave_scan(mine), 63);          // the host has seen to it that this fits
  longest = (int)__builtin_amdgcn_readlane(wave_max_up((unsigned)longest), 63);
  const FragmentRule rule = BITS4 ? bits4_fragment_rule(total, longest, heads, Q.tokens * Q.group, Q.target, C.slot_stride > ROW4)
                                  : fragment_rule(total, longest, heads, Q.tokens * Q.group, Q.target);
  int before = 0;
  for (int h0 = 0; h0 < heads; h0 += 64 * SCAN_GROUP) {
    if (h0 > 0) fetch(h0);
#pragma unroll
    for (int i = 0; i < SCAN_GROUP; ++i) {
      if (i > 0 && h0 + 64 * i >= heads) break;
      const int steps = steps_at(h0, i);
      const int parts = fragments_of(steps, rule);
      const int upto = before + wave_scan(parts);
      const unsigned long long beyond = __ballot(upto > fragment);
      if (beyond != 0) {
        int at = __builtin_ctzll(beyond);
        const int each = rule.per > 0 ? rule.per : 1 << rule.log;
        int k = -1;                                  // the part, where it is not the fragment's place
        if (BITS4) {
          const int two = at & ~1, p0 = __builtin_amdgcn_readlane(parts, two), p1 = __builtin_amdgcn_readlane(parts, two | 1);
          const int start = __builtin_amdgcn_readlane(upto, two) - p0, q = fragment - start, both = 2 * min(p0, p1);
          at = two | (q < both ? q & 1 : p1 > p0 ? 1 : 0);
          k = q < both ? q >> 1 : q - (both >> 1);
        }
        F.head = h0 + 64 * i + at;
        F.count = __builtin_amdgcn_readlane(size[i].count, at);
        F.n = __builtin_amdgcn_readlane(size[i].n, at);
        F.parts = __builtin_amdgcn_readlane(parts, at);
        F.first = __builtin_amdgcn_readlane(upto, at) - F.parts;
        if (BITS4)
          fragment = F.first + k;
        else
          k = fragment - F.first;
        F.step0 = k * each;
        F.step1 = min(F.step0 + each, __builtin_amdgcn_readlane(steps, at));
        return true;
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
  }
  return false;
}

// Part blockIdx.x / heads of a head.  Workgroups go round the eight XCDs, and heads often come in eights: neighbours in a group of eight
// change places from group to group, or an XCD would have the same kv head of every request, long or short.
template <bool BITS4 = false>
__device__ __forceinline__ bool split_part(const CacheView &C, const Queries &Q, Fragment &F, int &fragment) {
  const unsigned heads = (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads;
  const unsigned part = Q.split == 1 ? 0u : blockIdx.x / heads, i = blockIdx.x - part * heads;
  if (BITS4)
    F.head = (int)((i | 15u) < heads ? (i & ~15u) | (((i + (i >> 4) + part) & 7u) << 1) | (i >> 3 & 1u) : i);
  else
    F.head = (int)((i | 7u) < heads ? (i & ~7u) | ((i + (i >> 3) + part) & 7u) : i);
  const HeadSize size = head_size(C, Q, (unsigned)F.head);
  F.count = size.count;
  F.n = size.n;
  const int steps = steps_of(size.count, size.n);
  const int per = Q.split == 1 ? steps : max(1 << ATT_LEAST_LOG, (int)((unsigned)(steps + Q.split - 1) / (unsigned)Q.split));
  F.first = F.head * Q.split;
  F.parts = Q.split == 1 ? 1 : (int)((unsigned)(steps + per - 1) / (unsigned)per);
  F.step0 = (int)part * per;
  F.step1 = min(F.step0 + per, steps);
  fragment = F.first + (int)part;
  return (int)part < F.parts;
}

// The tiles of a part that a wave has: every wave a run of them.
struct Run { int begin, end, first, tiles; };
__device__ __forceinline__ Run run_of(const Fragment &part, int wave) {
  Run u;
  u.end = part.n > 0 ? min(part.step1 * ATT_STEP, part.count) : 0;      // no queries: no tiles
  u.begin = part.step0 * ATT_STEP;
  const int each = (max(u.end - u.begin, 0) + ATT_STEP - 1) / ATT_STEP;
  u.first = u.begin + wave * each * ATT_TILE;
  u.tiles = u.first < u.end ? min(each, (u.end - u.first + ATT_TILE - 1) / ATT_TILE) : 0;
  return u;
}


// Query rows as B operands: lane l has row l & 15, channels 32 kk + 8 (l >> 4) .. (GROUPS: 32 (l >> 4) + 8 kk ..); see: the slots that it sees.
template <int NT, bool GROUPS = false>
__device__ __forceinline__ void load_queries(const Queries &Q, const HeadOf &w, int R, int count, int n, Piece (&q)[NT][4], int (&see)[NT]) {
  const int n16 = threadIdx.x & 15, j = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 16 * nt + n16, t = r / Q.group;
    see[nt] = r < R ? sees(count, n, t) : 0;
    const uint16_t *qp = Q.q + w.b * Q.q_stride_b + w.l * Q.q_stride_l + t * Q.q_stride_t + (w.h * Q.group + r - t * Q.group) * Q.q_stride_h;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      q[nt][kk].u = make_uint4(0, 0, 0, 0);
      if (see[nt] > 0) q[nt][kk].u = *reinterpret_cast<const uint4 *>(GROUPS ? qp + 32 * j + 8 * kk : qp + 32 * kk + 8 * j);
    }
  }
}

// How products of K with query rows become logits in base 2.
struct Scaling {
  bool capped;
  float to_base2, to_y, cap2;
};
__device__ __forceinline__ Scaling scaling_of(const Queries &Q) {
  const bool capped = Q.softcap > 0.f;
  return Scaling{capped, Q.scale * LOG2E, capped ? Q.scale / Q.softcap : 0.f, Q.softcap * LOG2E};
}
// tanh(y) = 1 - 2 / (e^2y + 1); near 0, where that cancels, y times a polynomial in y^2
__device__ __forceinline__ float capped_small(const Scaling &c, float dot) {         // |y| < 1/4
  const float y = dot * c.to_y, z = y * y;
  const float slope = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  return dot * c.to_base2 * slope;
}
__device__ __forceinline__ float capped_logit(const Scaling &c, float dot) {
  const float y = dot * c.to_y;
  const float far = c.cap2 - 2.f * c.cap2 * __builtin_amdgcn_rcpf(exp2_(y * (2.f * LOG2E)) + 1.f);
  return y * y < 1.f / 16.f ? capped_small(c, dot) : far;
}

// Where the maximum is -inf the sum is 0 (nothing was seen) or NaN (only logits that are none), which stays.
__device__ __forceinline__ void add_stats(float &m, float &l, const float2 &x) {
  const float to = fmaxf(m, x.x);
  l = to == -INFINITY ? l + x.y : l * exp2_(m - to) + x.y * exp2_(x.x - to);
  m = to;
}

// Maximum and sum of row r over the fragments, by the lanes of a wave.
__device__ __forceinline__ float2 join_stats(const Queries &Q, int first, int parts, int R, int r) {
  float m = -INFINITY, l = 0.f;
  for (int k = threadIdx.x & 63; k < parts; k += 64) add_stats(m, l, Q.stats[(long long)(first + k) * R + r]);
  float top = m;
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = top == -INFINITY ? l : l * exp2_(m - top);
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  return make_float2(top, sum);
}

// What every row's weights are relative to, by a workgroup; stats: 256 entries; *none is 0 to all of it.
__device__ __forceinline__ void row_sums(const Queries &Q, const Fragment &f, int R, float2 *stats, float *lse2, int *none) {
  const int tid = threadIdx.x;
  // Up to 16 rows the waves take rows in turn, their lanes fragments (4 rows, 2.3 M slots: 248 us a call, in the other way 250);
  // more of them all at once: thread (group, row) takes every groups-th fragment, the first R threads add up the groups' (28 rows,
  // 72 heads of up to 3618: 56 us a call, in the first way 60).
  if (R <= 16) {
    for (int r = tid >> 6; r < R; r += 4) {
      const float2 all = join_stats(Q, f.first, f.parts, R, r);
      if ((tid & 63) == 0) lse2[r] = weights_from(Q, f.count, f.n, r, all.x, all.y, none);
    }
  } else {
    const int groups = (int)(256u / (unsigned)R), group = (int)((unsigned)tid / (unsigned)R), r = tid - group * R;
    float m = -INFINITY, l = 0.f;
    if (group < groups)
      for (int k = group; k < f.parts; k += groups) add_stats(m, l, Q.stats[(long long)(f.first + k) * R + r]);
    stats[tid] = make_float2(m, l);
    __syncthreads();
    if (tid < R) {
#pragma unroll 4
      for (int i = 1; i < min(groups, f.parts); ++i) add_stats(m, l, stats[i * R + tid]);
      lse2[tid] = weights_from(Q, f.count, f.n, tid, m, l, none);
    }
  }
}

// The four waves of a workgroup meet: rows of its only fragment are finished, else what the fragment has of them goes into the workspace.
// A wave's lane has sums of query 16 nt + (l & 15) (m: what its exponents are relative to, l: the lane's part of the weights' sum), acc[nt][c][vv]
// of channel 32 (l >> 4) + 8 vv + c.  Lds: o, m, l, lse2 and none, which is 0.
template <int NT, class Lds>
__device__ __forceinline__ void waves_meet(const CacheView &C, const Queries &Q, const HeadOf &w, const Fragment &part, int fragment, Lds &L,
                                           f32x4 (&acc)[NT][8], float (&m)[NT], float (&l)[NT], const int (&see)[NT]) {
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, j = lane >> 4;
  const int R = Q.tokens * Q.group;
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
    for (int i = 0; i < ATT_WAVES; ++i) sum += mm == -INFINITY ? L.l[i][row] : L.l[i][row] * exp2_(L.m[i][row] - mm);     // (-inf: 0, or NaN)
    f32x4 o[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      o[c] = *reinterpret_cast<const f32x4 *>(&L.o[0][tid >> 4][ch + 4 * c]);
#pragma unroll
      for (int i = 1; i < ATT_WAVES; ++i) o[c] += *reinterpret_cast<const f32x4 *>(&L.o[i][tid >> 4][ch + 4 * c]);
    }
    if (row < R) {
      if (part.parts == 1) {
        finish_row(C, Q, w, row, ch, o, mm, sum);
        if (ch == 0) L.lse2[row] = weights_from(Q, part.count, part.n, row, mm, sum, &L.none);
        if (ch == 0 && Q.weights != nullptr) Q.stats[(long long)fragment * R + row] = make_float2(mm, sum);
      } else {
        const long long at = (long long)fragment * R + row;
        f32x4 *to = reinterpret_cast<f32x4 *>(Q.partial + at * D + ch);
        to[0] = o[0];
        to[1] = o[1];
        if (ch == 0) Q.stats[at] = make_float2(mm, sum);
      }
    }
  }
}

// A workgroup that has all of a head adds its weights to the mass.
__device__ __forceinline__ void mass_here(const CacheView &C, const Queries &Q, const HeadPlace &hp, const float *logits, int R, int count,
                                          const float *lse2, const int *none) {
  __threadfence_block();
  __syncthreads();                                // the workgroup's logits and sums
  for (int at = 4 * (int)threadIdx.x; at < count; at += 4 * 256) {
    MassQuad M;
    mass_fetch(C, Q, hp, logits, R, at, count, M);
    mass_add(Q, lse2, *none, logits, R, at, M);
  }
}

// Lane n16 < 8 gets the n16-th of eight sums over 16 lanes: neighbours, pairs, fours, eights.
__device__ __forceinline__ float lanes_sum(const float (&sum)[8], int n16) {
  float mine = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y = sum[i];
    y += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0xb1, 0xf, 0xf, false));
    y += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x4e, 0xf, 0xf, false));
    y += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x141, 0xf, 0xf, false));
    y += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), 0x140, 0xf, 0xf, false));
    mine = n16 == i ? y : mine;
  }
  return mine;
}

// Weights of a fragment's slots, summed over the rows, to their mass.
__device__ __forceinline__ void weights_to_mass(const CacheView &C, const Queries &Q, const HeadPlace &hp, const float *weights, const Run &run,
                                                const int *none) {
  __threadfence_block();
  __syncthreads();
  const float inv = 1.f / (float)Q.group;
  for (int at = run.begin + 4 * (int)threadIdx.x; at < run.end; at += 4 * 256) {
    MassQuad M;
    mass_fetch(C, Q, hp, weights, 1, at, run.end, M);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (M.there[i]) *M.mass[i] = at + i < *none ? NAN : fmaf(M.x[0][i], inv, M.old[i]);
  }
}

// A call, checked and planned (cache_attention.hip), with the kernels of one kind of rows.  row16: pages hold whole halves of tiles, see there.
struct AttendKernels {
  void (*attend)(const CacheView &C, const Queries &Q, bool row16, unsigned blocks, hipStream_t st);
  void (*mass)(const CacheView &C, const Queries &Q, bool row16, unsigned blocks, hipStream_t st);
  bool bits4;                  // fragments by bits4_fragment_rule
  int again_rows;              // weights of more rows, with logits of more bytes, are found from K
  size_t again_bytes;
};
int attend_workspace(const CacheView &C, const compactor_cache_query_t *query, const AttendKernels &kernels, size_t *bytes);
int attend_call(const CacheView &C, const compactor_cache_query_t *query, const AttendKernels &kernels, bool row16, void *workspace,
                size_t workspace_bytes, void *stream);

}  // namespace cmp
