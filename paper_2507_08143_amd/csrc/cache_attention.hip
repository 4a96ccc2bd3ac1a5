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
#include <math.h>

#include <algorithm>
#include <type_traits>

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

// Steps of ATT_STEP slots of a head: one at least, so that every head has a workgroup that writes its rows.
__device__ __forceinline__ int steps_of(int count, int n) { return n > 0 && count > ATT_STEP ? (int)(((unsigned)count + ATT_STEP - 1) / ATT_STEP) : 1; }
struct HeadSize { int count, n; };           // tokens held, and queries
__device__ __forceinline__ HeadSize head_size(const CacheView &C, const Queries &Q, unsigned g) {
  const HeadOf w = head_of(C, g);
  return HeadSize{held(C, w.b, w.l, w.h), tokens_new(Q.new_tokens, w.b, Q.tokens)};
}

// How long a head is only the device knows, so up to SCAN_HEADS heads every wave finds its workgroup's part by itself, without a
// barrier: heads are cut into fragments of the same power of two of steps, numbered head after head, at most `target` of them beside
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
__device__ __forceinline__ bool scan_part(const CacheView &C, const Queries &Q, int fragment, Fragment &F) {
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
  const FragmentRule rule = fragment_rule(total, longest, heads, Q.tokens * Q.group, Q.target);
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
        const int at = __builtin_ctzll(beyond), each = rule.per > 0 ? rule.per : 1 << rule.log;
        F.head = h0 + 64 * i + at;
        F.count = __builtin_amdgcn_readlane(size[i].count, at);
        F.n = __builtin_amdgcn_readlane(size[i].n, at);
        F.parts = __builtin_amdgcn_readlane(parts, at);
        F.first = __builtin_amdgcn_readlane(upto, at) - F.parts;
        F.step0 = (fragment - F.first) * each;
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
__device__ __forceinline__ bool split_part(const CacheView &C, const Queries &Q, Fragment &F, int &fragment) {
  const unsigned heads = (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads;
  const unsigned part = Q.split == 1 ? 0u : blockIdx.x / heads, i = blockIdx.x - part * heads;
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

// Query rows as B operands: lane l has row l & 15, channels 32 kk + 8 (l >> 4) ..; see: the slots that it sees.
template <int NT>
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
      if (see[nt] > 0) q[nt][kk].u = *reinterpret_cast<const uint4 *>(qp + 32 * kk + 8 * j);
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
__device__ __forceinline__ float capped_logit(const Scaling &c, float dot) {
  const float y = dot * c.to_y, z = y * y;
  const float far = c.cap2 - 2.f * c.cap2 * __builtin_amdgcn_rcpf(exp2_(y * (2.f * LOG2E)) + 1.f);
  const float slope = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  return z < 1.f / 16.f ? dot * c.to_base2 * slope : far;
}

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
      if (complete) {
        finish_row(C, Q, w, row, ch, o, mm, sum);
        if (ch == 0) L.lse2[row] = weights_from(Q, count, n, row, mm, sum, &L.none);
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
  if (kept_in_lds<NT> && store && tiles > 0) leave(tiles);
  if (complete && store && n > 0) {
    __threadfence_block();
    __syncthreads();                                // the workgroup's logits and sums
    for (int at = 4 * tid; at < count; at += 4 * 256) {
      MassQuad M;
      mass_fetch(C, Q, hp, logits, R, at, count, M);
      mass_add(Q, L.lse2, L.none, logits, R, at, M);
    }
  }
}

// Second launch: the fragments of a head meet.  The first heads * R workgroups take a query row each, 16 fragments side by side
// and 8 channels a thread; the others add a fragment's weights to the mass.

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

__global__ __launch_bounds__(256) void attend_join_kernel(const CacheView C, const Queries Q) {
  __shared__ float part_o[16][D + 4], lse2[MOST_ROWS];
  __shared__ float2 stats[256];                     // of the groups of more than 16 rows
  __shared__ int none;
  const int tid = threadIdx.x, R = Q.tokens * Q.group;
  const unsigned rows = (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads * (unsigned)R;
  if (blockIdx.x < rows) {
    const unsigned g = blockIdx.x / (unsigned)R;
    const int r = (int)(blockIdx.x - g * (unsigned)R);
    const int2 f = Q.head_frags[g];
    if (f.y < 2) return;                            // its only workgroup has finished it
    const float2 all = join_stats(Q, f.x, f.y, R, r);      // (every wave)
    const int sl = tid >> 4, ch = 8 * (tid & 15);
    f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    for (int k = sl; k < f.y; k += 16) {
      const long long at = (long long)(f.x + k) * R + r;
      const float mk = Q.stats[at].x, scale = all.x == -INFINITY ? 0.f : exp2_(mk - all.x);
      const f32x4 *x = reinterpret_cast<const f32x4 *>(Q.partial + at * D + ch);
      o[0] += x[0] * scale;
      o[1] += x[1] * scale;
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
  const Fragment f = Q.frags[blockIdx.x - rows];
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
    // over the 16 lanes: neighbours, pairs, fours, eights
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
    if (n16 < 8) weights[s0 + 16 * (n16 >> 2) + 4 * j + (n16 & 3)] = mine;
    there = there_next;
    __builtin_amdgcn_sched_barrier(0);
  };
  if (tiles > 0) {
    for (int tile = 0; tile + 1 < tiles; ++tile) one_tile(tile, std::true_type());
    one_tile(tiles - 1, std::false_type());
  }
  __threadfence_block();
  __syncthreads();
  const float inv = 1.f / (float)Q.group;
  for (int at = run.begin + 4 * tid; at < run.end; at += 4 * 256) {
    MassQuad M;
    mass_fetch(C, Q, hp, weights, 1, at, run.end, M);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (M.there[i]) *M.mass[i] = at + i < none ? NAN : fmaf(M.x[0][i], inv, M.old[i]);
  }
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

static AttendPlan attend_plan(const CacheView &C, const compactor_cache_query_t *q) {
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
    A.target = fragment_target(heads, steps, A.rows, cus);
    A.frags_most = fragments_most((int)heads, A.target);
  } else if (steps > ATT_ALONE) {
    A.split = (int)std::max(std::min(std::min(SPLIT_ALL / heads, (long long)SPLIT_MOST), ((steps - 1) >> ATT_LEAST_LOG) + 1), 1ll);
    if (A.split > 1) A.frags_most = A.split * (int)heads;
  }
  A.joined = A.frags_most > 0;
  A.pitch = (int)((most + ATT_TILE - 1) / ATT_TILE * ATT_TILE);
  const size_t a_row = (size_t)heads * A.pitch * sizeof(float);
  A.again = q->accumulate && A.rows > AGAIN_ROWS && a_row * A.rows > AGAIN_BYTES;
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
  if (!query->q || !query->out || query->out == query->q) return COMPACTOR_EINVAL;
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
  const long long blocks = A.frags_most > 0 ? A.frags_most : heads;
  const long long join = A.joined ? heads * A.rows + (query->accumulate && !A.again ? A.frags_most : 0) : 0;
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
  // halves of tiles with one origin, and offsets inside one that fit 32 bits
  const bool page16 = C.page_size % 16 == 0 && C.slot_stride <= (1 << 24);
  if (page16)
    launch_attend<true>(C, Q, (unsigned)blocks, st);
  else
    launch_attend<false>(C, Q, (unsigned)blocks, st);
  if (A.joined) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    hipLaunchKernelGGL(attend_join_kernel, dim3((unsigned)join), dim3(256), 0, st, C, Q);
  }
  if (A.again) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    const auto kernel = A.rows <= 48 ? (page16 ? attend_mass_kernel<3, true> : attend_mass_kernel<3, false>)
                                     : (page16 ? attend_mass_kernel<4, true> : attend_mass_kernel<4, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, C, Q);
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
