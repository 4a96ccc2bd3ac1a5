// The cache in 4 bits beside one in 16: its making from one (store) and its rows as bf16 (read).  Rows in (append) and out (eviction):
// cache.hip; attention: fp4_attention.hip.
#include "fp4.h"

namespace cmp {

// ------------------------------------------------------------------------------------------ store
// 16 lanes take a row of K and of V, 8 channels a lane.  Bound by HBM: 512 bytes a token in, 136 out, 16 of mass and position; 2.5 M tokens of 12
// requests in 336 us, 4.9 TB/s, which is what a copy reaches.
constexpr int STORE_ROWS = 64;       // of a head per workgroup and step
// Workgroups, beside one a head.  How many rows there are only the device knows, and tables often have room for many more, so a head's workgroups step through its rows
// (16 requests of 256 heads that hold 1000 tokens, tables for 131 072 each: 8905 us with a workgroup for every 64 that there is room for, 556 with these).
constexpr long long STORE_MOST = 65536;

__global__ __launch_bounds__(256) void store_kernel(const CacheView T, const CacheView S, int parts) {
  const unsigned g = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - g * (unsigned)parts), lane = threadIdx.x & 15;
  const HeadOf w = head_of(T, g);
  const int count = held(S, w.b, w.l, w.h), room = min(count, T.capacity);
  if (part == 0 && threadIdx.x == 0) {
    T.counts[count_at(T, w.b, w.l, w.h)] = room;
    if (T.seen != nullptr) T.seen[count_at(T, w.b, w.l, w.h)] = S.seen[count_at(S, w.b, w.l, w.h)];
  }
  const HeadPlace from = head_place(S, w), to = head_place(T, w);
  for (int slot0 = part * STORE_ROWS; slot0 < room; slot0 += parts * STORE_ROWS) {
#pragma unroll
    for (int i = 0; i < STORE_ROWS / 16; ++i) {
      const int slot = slot0 + 16 * i + (int)(threadIdx.x >> 4);
      if (slot >= room) break;
      const SlotPlace a = slot_place(S, from, slot), z = slot_place(T, to, slot);
      if (!page_there(S, a.page) || !page_there(T, z.page)) continue;      // (the same for the 16 lanes)
      const long long src = row_at(S, from, a) + 8 * lane, dst = row_at(T, to, z) + 2 * lane;
      const uint4 k = load_stream16(S.k + src), v = load_stream16(S.v + src);
      uint32_t k_scales, v_scales;
      *reinterpret_cast<unsigned *>(T.k + dst) = fp4_encode_row(k, lane, k_scales);
      *reinterpret_cast<unsigned *>(T.v + dst) = fp4_encode_row(v, lane, v_scales);
      if (lane == 0) {
        const long long y = state_at(T, to, z);
        T.k_scales[y] = k_scales;
        T.v_scales[y] = v_scales;
        if (T.mass != nullptr) {
          const long long x = state_at(S, from, a);
          T.mass[y] = S.mass[x];
          T.positions[y] = S.positions[x];
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------ read
struct RowsOut {
  uint16_t *k, *v;
  long long stride_b, stride_l, stride_t, stride_h;
  const int32_t *new_tokens;
  int tokens, first;
};
// The same the other way: 136 bytes a token in, 512 out, 2.5 M tokens in 328 us, 5.0 TB/s; the last token of 96 heads 3.4 us, most of which is the launch.
constexpr int READ_ROWS = 64;        // of a head per workgroup

__global__ __launch_bounds__(256) void read_kernel(const CacheView C, const RowsOut R, int parts) {
  const unsigned g = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - g * (unsigned)parts), lane = threadIdx.x & 15;
  const HeadOf w = head_of(C, g);
  const HeadPlace p = head_place(C, w);
  const int n = tokens_new(R.new_tokens, w.b, R.tokens), count = held(C, w.b, w.l, w.h);
  const long long first = R.first >= 0 ? R.first : (long long)count - n;
#pragma unroll
  for (int i = 0; i < READ_ROWS / 16; ++i) {
    const long long t = (long long)part * READ_ROWS + 16 * i + (threadIdx.x >> 4), slot = first + t;
    if (t >= R.tokens) return;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (t < n && slot >= 0 && slot < count) {
      const SlotPlace s = slot_place(C, p, (int)slot);
      if (page_there(C, s.page)) {
        const long long src = row_at(C, p, s) + 2 * lane, at = state_at(C, p, s);
        k = fp4_decode(*reinterpret_cast<const unsigned *>(C.k + src), fp4_scale(C.k_scales[at], lane >> 2));
        v = fp4_decode(*reinterpret_cast<const unsigned *>(C.v + src), fp4_scale(C.v_scales[at], lane >> 2));
      }
    }
    const long long dst = w.b * R.stride_b + w.l * R.stride_l + t * R.stride_t + w.h * R.stride_h + 8 * lane;
    store_stream16(R.k + dst, k);
    store_stream16(R.v + dst, v);
  }
}

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_mx_store(const compactor_mx_cache_t *cache, const compactor_cache_t *source, void *stream) {
  CacheView T, S;
  int rc = cache_view(cache, CACHE_ROWS, &T);
  if (rc) return rc;
  rc = cache_view(source, T.mass != nullptr ? CACHE_STATE : CACHE_ROWS, &S);
  if (rc) return rc;
  if (T.nreq != S.nreq || T.layers != S.layers || T.kv_heads != S.kv_heads) return COMPACTOR_EINVAL;
  if (T.counts == S.counts || T.k == S.k || T.v == S.v || T.k == S.v || T.v == S.k) return COMPACTOR_EINVAL;
  const long long heads = (long long)T.nreq * T.layers * T.kv_heads;
  const int parts = (int)min((min(T.capacity, S.capacity) + STORE_ROWS - 1ll) / STORE_ROWS, max(STORE_MOST / heads, 1ll));
  if (!launchable(heads * parts, 256)) return COMPACTOR_EINVAL;
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(store_kernel, dim3((unsigned)(heads * parts)), dim3(256), 0, static_cast<hipStream_t>(stream), T, S, parts);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

int compactor_mx_read(const compactor_mx_cache_t *cache, const compactor_cache_rows_out_t *rows, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_ROWS, &C);
  if (rc) return rc;
  if (!rows || !rows->k || !rows->v || rows->k == rows->v || rows->tokens < 1 || rows->first < -1) return COMPACTOR_EINVAL;
  if (rows->stride_b < 0 || rows->stride_l < 0 || rows->stride_t < 0 || rows->stride_h < 0) return COMPACTOR_EINVAL;
  if (((reinterpret_cast<uintptr_t>(rows->k) | reinterpret_cast<uintptr_t>(rows->v)) & 15u) ||
      ((rows->stride_b | rows->stride_l | rows->stride_t | rows->stride_h) & 7) || (reinterpret_cast<uintptr_t>(rows->new_tokens) & 3u))
    return COMPACTOR_EALIGN;
  const RowsOut R{static_cast<uint16_t *>(rows->k), static_cast<uint16_t *>(rows->v), rows->stride_b, rows->stride_l, rows->stride_t,
                  rows->stride_h, rows->new_tokens, rows->tokens, rows->first};
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  const int parts = (int)(((long long)R.tokens + READ_ROWS - 1) / READ_ROWS);
  if (!launchable(heads * parts, 256)) return COMPACTOR_EINVAL;
  (void)hipGetLastError();
  hipLaunchKernelGGL(read_kernel, dim3((unsigned)(heads * parts)), dim3(256), 0, static_cast<hipStream_t>(stream), C, R, parts);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
