// What the kernels that serve from a paged cache share: the cache as a launch sees it, and where its
// slots lie (see compactor_cache_t).
#pragma once

#include "common.h"

namespace cmp {

struct CacheView {
  uint16_t *k, *v;
  long long page_stride, layer_stride, head_stride, slot_stride;   // elements
  const int32_t *tables;
  long long table_stride;
  int page_size, num_pages, capacity;        // capacity: slots that a table names
  unsigned div_mul, div_shift;               // slot / page_size, see invariant_quotient()
  unsigned req_mul, req_shift, layer_mul, layer_shift;      // head / (layers * kv_heads), head / kv_heads
  int nreq, layers, kv_heads;
  int32_t *counts, *seen;
  long long count_stride_b, count_stride_l;
  float *mass;
  int32_t *positions;
  long long state_page_stride, state_layer_stride, state_head_stride;
  uint32_t *k_scales, *v_scales;             // rows of 4 bits: their scales, at the place of mass; else null
};
constexpr int ROW4 = D / 4;                  // a row of 4 bits in the units of the strides above

// x / d for 0 <= x < 2^31, by the multiplicative inverse of an invariant divisor (Granlund and Montgomery 1994): with
// 2^(shift-1) < d <= 2^shift and mul = floor(2^32 (2^shift - d) / d) + 1 the quotient is (mulhi(x, mul) + x) >> shift, and the
// sum stays below 2^32 because mulhi(x, mul) <= x.  (A division takes some 30 instructions before a first load.)
__host__ __device__ __forceinline__ int invariant_quotient(unsigned x, unsigned mul, unsigned shift) {
  const unsigned hi = (unsigned)(((unsigned long long)x * mul) >> 32);
  return (int)((hi + x) >> shift);
}
inline void invariant_divisor(int d, unsigned *mul, unsigned *shift) {
  unsigned s = 0;
  while ((1ull << s) < (unsigned long long)d) ++s;
  *shift = s;
  *mul = (unsigned)((((1ull << s) - (unsigned long long)d) << 32) / (unsigned long long)d + 1);
}

__device__ __forceinline__ long long count_at(const CacheView &C, int b, int l, int h) {
  return b * C.count_stride_b + l * C.count_stride_l + h;
}
__device__ __forceinline__ int clamp_to(int x, int most) { return x < 0 ? 0 : (x < most ? x : most); }
__device__ __forceinline__ int held(const CacheView &C, int b, int l, int h) {
  return clamp_to(C.counts[count_at(C, b, l, h)], C.capacity);
}
// New tokens of a request, of T rows.
__device__ __forceinline__ int tokens_new(const int32_t *new_tokens, int b, int T) {
  if (new_tokens == nullptr) return T;
  return clamp_to(new_tokens[b], T);
}
__device__ __forceinline__ bool page_there(const CacheView &C, int page) { return (unsigned)page < (unsigned)C.num_pages; }

// Head (b, l, h) of launch-wide number g.
struct HeadOf { int b, l, h; };
__device__ __forceinline__ HeadOf head_of(const CacheView &C, unsigned g) {
  HeadOf w;
  w.b = invariant_quotient(g, C.req_mul, C.req_shift);
  const unsigned r = g - (unsigned)w.b * ((unsigned)C.layers * (unsigned)C.kv_heads);
  w.l = invariant_quotient(r, C.layer_mul, C.layer_shift);
  w.h = (int)(r - (unsigned)w.l * (unsigned)C.kv_heads);
  return w;
}

// The parts of the places of a head's slots that do not depend on the slot.
struct HeadPlace {
  const int32_t *table;
  long long rows, state;       // of (l, h), in elements of the pages and of mass and positions
};
__device__ __forceinline__ HeadPlace head_place(const CacheView &C, const HeadOf &w) {
  return HeadPlace{C.tables + w.b * C.table_stride, w.l * C.layer_stride + w.h * C.head_stride,
                   w.l * C.state_layer_stride + w.h * C.state_head_stride};
}
// A slot's page (may not be there) and place in it.
struct SlotPlace { int page, at; };
__device__ __forceinline__ SlotPlace slot_place(const CacheView &C, const HeadPlace &p, int slot) {
  const int i = invariant_quotient((unsigned)slot, C.div_mul, C.div_shift);
  return SlotPlace{p.table[i], slot - i * C.page_size};
}
__device__ __forceinline__ long long row_at(const CacheView &C, const HeadPlace &p, const SlotPlace &s) {
  return s.page * C.page_stride + p.rows + s.at * C.slot_stride;
}
__device__ __forceinline__ long long state_at(const CacheView &C, const HeadPlace &p, const SlotPlace &s) {
  return s.page * C.state_page_stride + p.state + s.at;
}

// The counts of a head that n tokens have been appended to.
__device__ __forceinline__ void append_count(const CacheView &C, const HeadOf &w, int count, int seen, int n) {
  const long long at = count_at(C, w.b, w.l, w.h);
  C.counts[at] = n < C.capacity - count ? count + n : C.capacity;
  if (C.seen != nullptr) C.seen[at] = (int)((unsigned)seen + (unsigned)n);
}

// Sum over the lanes up to this one (row shifts, then the sums of rows and of halves of the wave handed on).
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The largest of the lanes' numbers, in lane 63.
__device__ __forceinline__ unsigned wave_max_up(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
  return x;
}

// Whether a launch has fewer than 2^32 threads, the most that HIP takes.  Checked before a call's first launch.
inline bool launchable(long long blocks, int threads) { return blocks <= 0xffffffffll / threads; }

// Checks a caller's cache (COMPACTOR_OK or an error) and makes the view of it.
// sizes only; tables and counts; pages and counts; and seen, mass, positions
enum CacheNeed { CACHE_SIZES, CACHE_TABLES, CACHE_ROWS, CACHE_STATE };
int cache_view(const compactor_cache_t *c, CacheNeed need, CacheView *view);
int cache_view(const compactor_mx_cache_t *c, CacheNeed need, CacheView *view);       // rows of 4 bits

hipError_t launch_cache_admit(const SegTable &T, const CacheView &C, const int32_t *kept_idx, const int32_t *kept_cnt,
                              const float *scores, hipStream_t st);

}  // namespace cmp
