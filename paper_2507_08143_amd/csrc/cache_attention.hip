// Attention of new tokens to a paged cache (see compactor_cache_attention).
#include <math.h>

#include "cache.h"

namespace cmp {

struct Queries {
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  long long q_stride_b, q_stride_l, q_stride_t, q_stride_h;
  long long out_stride_b, out_stride_l, out_stride_t, out_stride_h;
  const int32_t *new_tokens;
  int tokens, group;           // T, and G query heads a kv head
  float scale, softcap;
  float *weights;              // [head][T * G][most]: p of every slot, or null
  int most;
};

__device__ __forceinline__ float bf16_float(uint16_t x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ uint16_t float_bf16(float x) {
  const __bf16 b = (__bf16)x;
  uint16_t u;
  __builtin_memcpy(&u, &b, 2);
  return u;
}

// A workgroup per query row: one pass for the maximum and the sum, one for the output.
__global__ __launch_bounds__(256) void attend_kernel(const CacheView C, const Queries Q) {
  __shared__ float q[D], red[2][256], p[256], acc[2][D];
  const int R = Q.tokens * Q.group, tid = threadIdx.x;
  const unsigned g = blockIdx.x / (unsigned)R;
  const int r = (int)(blockIdx.x - g * (unsigned)R), t = r / Q.group, j = r - t * Q.group;
  const HeadOf w = head_of(C, g);
  const HeadPlace hp = head_place(C, w);
  const int count = held(C, w.b, w.l, w.h), n = tokens_new(Q.new_tokens, w.b, Q.tokens);
  const int sees = t < n ? max(count - (n - 1 - t), 0) : 0;
  const int qh = w.h * Q.group + j;
  if (tid < D) q[tid] = bf16_float(Q.q[w.b * Q.q_stride_b + w.l * Q.q_stride_l + t * Q.q_stride_t + qh * Q.q_stride_h + tid]);
  __syncthreads();
  auto logit = [&](int s) {
    const SlotPlace at = slot_place(C, hp, s);
    if (!page_there(C, at.page)) return -INFINITY;
    const uint16_t *k = C.k + row_at(C, hp, at);
    float x = 0.f;
    for (int c = 0; c < D; ++c) x = fmaf(q[c], bf16_float(k[c]), x);
    x *= Q.scale;
    return Q.softcap > 0.f ? Q.softcap * tanhf(x / Q.softcap) : x;
  };
  float m = -INFINITY, l = 0.f;
  for (int s = tid; s < sees; s += 256) m = fmaxf(m, logit(s));
  red[0][tid] = m;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if (tid < d) red[0][tid] = fmaxf(red[0][tid], red[0][tid + d]);
    __syncthreads();
  }
  m = red[0][0] == -INFINITY ? 0.f : red[0][0];
  const bool store = Q.weights != nullptr && count <= Q.most;
  float *weights = store ? Q.weights + ((long long)g * R + r) * Q.most : nullptr;
  float o = 0.f;
  for (int s0 = 0; s0 < count; s0 += 256) {
    const int s = s0 + tid;
    p[tid] = s < sees ? expf(logit(s) - m) : 0.f;
    l += p[tid];
    if (store && s < count) weights[s] = p[tid];
    __syncthreads();
    for (int i = tid >> 7; i < min(256, sees - s0); i += 2) {
      const SlotPlace at = slot_place(C, hp, s0 + i);
      if (page_there(C, at.page)) o = fmaf(p[i], bf16_float(C.v[row_at(C, hp, at) + (tid & 127)]), o);
    }
    __syncthreads();
  }
  red[1][tid] = l;
  acc[tid >> 7][tid & 127] = o;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if (tid < d) red[1][tid] += red[1][tid + d];
    __syncthreads();
  }
  l = red[1][0];
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (tid < D)
    Q.out[w.b * Q.out_stride_b + w.l * Q.out_stride_l + t * Q.out_stride_t + qh * Q.out_stride_h + tid] =
        float_bf16((acc[0][tid] + acc[1][tid]) * inv);
  if (tid == 0 && Q.lse != nullptr)
    Q.lse[(((long long)w.b * C.layers + w.l) * Q.tokens + t) * (C.kv_heads * Q.group) + qh] = l == 0.f ? -INFINITY : logf(l) + m;
  if (store)
    for (int s = tid; s < count; s += 256) weights[s] *= inv;
}

__global__ __launch_bounds__(256) void attend_mass_kernel(const CacheView C, const Queries Q) {
  const int R = Q.tokens * Q.group;
  const HeadOf w = head_of(C, blockIdx.x);
  const HeadPlace hp = head_place(C, w);
  const int count = held(C, w.b, w.l, w.h);
  if (count > Q.most) return;
  for (int s = threadIdx.x; s < count; s += 256) {
    const SlotPlace at = slot_place(C, hp, s);
    if (!page_there(C, at.page)) continue;
    float x = 0.f;
    for (int r = 0; r < R; ++r) x += Q.weights[((long long)blockIdx.x * R + r) * Q.most + s];
    C.mass[state_at(C, hp, at)] += x / (float)Q.group;
  }
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

static size_t query_bytes(const CacheView &C, const compactor_cache_query_t *q) {
  const size_t heads = (size_t)C.nreq * C.layers * C.kv_heads, rows = (size_t)q->tokens * (q->q_heads / C.kv_heads);
  return q->accumulate ? (heads * rows * query_most(C, q) * sizeof(float) + 255) / 256 * 256 : 0;
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
  *bytes = query_bytes(C, query);
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
  const size_t need = query_bytes(C, query);
  if (need > 0 && (!workspace || workspace_bytes < need)) return COMPACTOR_EWORKSPACE;
  if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return COMPACTOR_EALIGN;
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
  Q.weights = query->accumulate ? static_cast<float *>(workspace) : nullptr;
  Q.most = query_most(C, query);
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  if (heads * Q.tokens * Q.group > 0x7fffffffll) return COMPACTOR_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(attend_kernel, dim3((unsigned)(heads * Q.tokens * Q.group)), dim3(256), 0, st, C, Q);
  if (Q.weights != nullptr) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    hipLaunchKernelGGL(attend_mass_kernel, dim3((unsigned)heads), dim3(256), 0, st, C, Q);
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
