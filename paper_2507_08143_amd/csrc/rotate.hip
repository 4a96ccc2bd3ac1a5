// Norms and rotary positions of query and key heads (see compactor_rotate), alone and on the way into a cache.
//
// 16 lanes take a row of 128 channels, 8 a lane in two pieces of 4: for rotated lanes the first and second members of pairs 4 c .. 4 c + 3
// (interleaved: the 4 pairs themselves), so that no channel has to be fetched from another lane, and a lane's 4 sines and cosines serve
// all heads of a token.
#include "cache.h"
#include "fp4.h"

namespace cmp {

struct Rotation {
  const double *freqs;
  const float *q_norm, *k_norm;
  int turned, interleaved;         // lanes of a row that rotate
  float eps;
};

// A row as a lane sees it: where its two pieces begin.
struct RowPieces { int lo, hi; };
__device__ __forceinline__ RowPieces row_pieces(const Rotation &R, int lane) {
  if (R.interleaved || lane >= R.turned) return RowPieces{8 * lane, 8 * lane + 4};       // 8 R.turned is rotary_dim
  return RowPieces{4 * lane, 4 * R.turned + 4 * lane};
}

// Sine and cosine of p * freq: the angle in 64 bits, in quarter turns, what is left of it (an eighth of a turn at most) in fp32 by Taylor's
// series, cut where the next term is below 2^-29.  1 / 2 pi is the sum of two doubles: of an angle of 2^31 the turns are off by 2^-75.
struct Turn { float c[4], s[4]; };
__device__ __forceinline__ void turn_of(const Rotation &R, const double (&freqs)[4], int position, Turn &turn) {
  constexpr double INV_HI = 0.15915494309189535, INV_LO = -9.839338337591243e-18;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double a = (double)position * freqs[i];
    const double quarters = rint(a * (4.0 * INV_HI));
    const double rest = fma(a, 4.0 * INV_LO, fma(a, 4.0 * INV_HI, -quarters));             // of a quarter, -1/2 .. 1/2
    const int quadrant = (int)(quarters - 4.0 * floor(quarters * 0.25));
    const float x = (float)rest * 1.57079632679489662f, z = x * x;
    const float s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float cc = quadrant & 1 ? s : c, ss = quadrant & 1 ? c : s;
    turn.c[i] = quadrant == 1 || quadrant == 2 ? -cc : cc;
    turn.s[i] = quadrant & 2 ? -ss : ss;
  }
}
__device__ __forceinline__ void turn_freqs(const Rotation &R, int lane, double (&freqs)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) freqs[i] = lane < R.turned ? R.freqs[4 * lane + i] : 0.0;      // (lanes that do not rotate: by 0)
}

// Weights of a norm, the lane's 8 channels.
struct Weights { float w[8]; };
__device__ __forceinline__ void load_weights(const float *norm, int layer, const RowPieces &p, Weights &W) {
  const float *w = norm + (long long)layer * D;
  const float4 a = *reinterpret_cast<const float4 *>(w + p.lo), b = *reinterpret_cast<const float4 *>(w + p.hi);
  W = Weights{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

struct Raw { uint2 lo, hi; };      // 8 channels of bf16
__device__ __forceinline__ Raw load_raw(const uint16_t *row, const RowPieces &p) {
  return Raw{*reinterpret_cast<const uint2 *>(row + p.lo), *reinterpret_cast<const uint2 *>(row + p.hi)};
}
__device__ __forceinline__ void store_raw(uint16_t *row, const RowPieces &p, const Raw &x) {
  *reinterpret_cast<uint2 *>(row + p.lo) = x.lo;
  *reinterpret_cast<uint2 *>(row + p.hi) = x.hi;
}
__device__ __forceinline__ unsigned two_bf16(float a, float b) {
  bf16x2 t;
  t[0] = (__bf16)a;
  t[1] = (__bf16)b;
  unsigned u;
  __builtin_memcpy(&u, &t, 4);
  return u;
}
__device__ __forceinline__ Raw to_raw(const float (&y)[8]) {
  return Raw{make_uint2(two_bf16(y[0], y[1]), two_bf16(y[2], y[3])), make_uint2(two_bf16(y[4], y[5]), two_bf16(y[6], y[7]))};
}

// Over the 16 lanes of a row: neighbours, pairs, fours, eights.
__device__ __forceinline__ float row_sum(float x) {
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xb1, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4e, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xf, 0xf, false));
  return x;
}

// y of a row (see compactor_rotate_rows); by all 16 lanes
__device__ __forceinline__ void norm_row(const Raw &x, bool norm, const Weights &W, float eps, float (&y)[8]) {
  const unsigned w[4] = {x.lo.x, x.lo.y, x.hi.x, x.hi.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(w[i] << 16);
    y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  if (norm) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
    const float inv = __builtin_amdgcn_rsqf(fmaf(row_sum(sum), 1.f / D, eps));
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * inv * W.w[i];
  }
}
__device__ __forceinline__ Raw turn_row(const Rotation &R, const Turn &turn, bool turned, const float (&y)[8]) {
  float z[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = R.interleaved ? y[2 * i] : y[i], b = R.interleaved ? y[2 * i + 1] : y[4 + i];
    const float first = fmaf(a, turn.c[i], -(b * turn.s[i])), second = fmaf(b, turn.c[i], a * turn.s[i]);
    if (R.interleaved) {
      z[2 * i] = first;
      z[2 * i + 1] = second;
    } else {
      z[i] = first;
      z[4 + i] = second;
    }
  }
  // channels that stay do so even where they are no numbers (0 * inf)
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = turned ? z[i] : y[i];
  return to_raw(z);
}

// ------------------------------------------------------------------------------------------ rotate
struct RotateRows {
  const uint16_t *q, *k;
  uint16_t *q_out, *k_out, *k_plain;
  long long q_b, q_l, q_t, q_h, k_b, k_l, k_t, k_h, qo_b, qo_l, qo_t, qo_h, ko_b, ko_l, ko_t, ko_h, kp_b, kp_l, kp_t, kp_h;
  const int32_t *positions;
  long long position_stride_b;
  const int32_t *new_tokens;
  int layers, tokens, q_heads, kv_heads;
  int parts;                       // waves that share the heads of a token
  unsigned units;                  // (request, layer, token, part)
};
constexpr int HEADS_MOST = 1 << 20;
constexpr int ROTATE_AT_ONCE = 4;  // rows that 16 lanes have on their way

// A wave per token of a layer, or several; its four rows of 16 lanes take heads in turn.  Bound by HBM for a prompt: 32 + 8 heads of 32 768 tokens with norms,
// keys before the rotation too (738 MB in and out), 131 us or 5.6 TB/s, more than a copy reaches; by the latency of position, frequencies and rows for few
// tokens, 4.1 us up to 64 of them with 32 + 8 heads.
__global__ __launch_bounds__(256) void rotate_kernel(const Rotation R, const RotateRows S) {
  const unsigned unit = blockIdx.x * 4u + (threadIdx.x >> 6);
  if (unit >= S.units) return;
  const unsigned token = unit / (unsigned)S.parts;
  const int part = (int)(unit - token * (unsigned)S.parts);
  const unsigned bl = token / (unsigned)S.tokens;
  const int t = (int)(token - bl * (unsigned)S.tokens);
  const long long b = bl / (unsigned)S.layers, l = bl - (unsigned)b * (unsigned)S.layers;
  if (t >= tokens_new(S.new_tokens, (int)b, S.tokens)) return;
  const int lane = threadIdx.x & 15, first = part * 4 + (int)(threadIdx.x >> 4 & 3), step = 4 * S.parts;
  const RowPieces p = row_pieces(R, lane);
  const bool turned = lane < R.turned;
  double freqs[4];
  turn_freqs(R, lane, freqs);
  const int position = S.positions[b * S.position_stride_b + t];
  Turn turn;
  turn_of(R, freqs, position, turn);
  auto rows = [&](const uint16_t *from, long long from_h, uint16_t *to, long long to_h, uint16_t *plain, long long plain_h, int heads, const float *norm) {
    Weights W;
    if (norm != nullptr) load_weights(norm, (int)l, p, W);
    for (int h0 = first; h0 < heads; h0 += ROTATE_AT_ONCE * step) {
      Raw x[ROTATE_AT_ONCE];
#pragma unroll
      for (int i = 0; i < ROTATE_AT_ONCE; ++i)
        if (h0 + i * step < heads) x[i] = load_raw(from + (h0 + i * step) * from_h, p);
#pragma unroll
      for (int i = 0; i < ROTATE_AT_ONCE; ++i) {
        const int h = h0 + i * step;
        if (h >= heads) break;
        float y[8];
        norm_row(x[i], norm != nullptr, W, R.eps, y);
        if (plain != nullptr) store_raw(plain + h * plain_h, p, to_raw(y));
        store_raw(to + h * to_h, p, turn_row(R, turn, turned, y));
      }
    }
  };
  rows(S.q + b * S.q_b + l * S.q_l + t * S.q_t, S.q_h, S.q_out + b * S.qo_b + l * S.qo_l + t * S.qo_t, S.qo_h, nullptr, 0, S.q_heads, R.q_norm);
  rows(S.k + b * S.k_b + l * S.k_l + t * S.k_t, S.k_h, S.k_out + b * S.ko_b + l * S.ko_l + t * S.ko_t, S.ko_h,
       S.k_plain != nullptr ? S.k_plain + b * S.kp_b + l * S.kp_l + t * S.kp_t : nullptr, S.kp_h, S.kv_heads, R.k_norm);
}

// ------------------------------------------------------------------------------------------ append
struct RotateAppend {
  const uint16_t *k, *v, *q;
  uint16_t *q_out;
  long long stride_b, stride_l, stride_t, stride_h;
  long long q_b, q_l, q_t, q_h, qo_b, qo_l, qo_t, qo_h;
  const int32_t *new_tokens;
  int tokens, group;               // query heads a kv head, 0: no queries
  int head_rows;                   // rows of 16 lanes a head has, 16 / that heads a workgroup
  int token_rows;                  // of them a token has
  int part, parts;                 // tokens of a head a workgroup takes, workgroups a head
};

// K, V and the G queries of a token of a head are G + 2 rows with one turn.  Bound by the latency of the chain count, table entry, row in small calls (one
// token of 512 heads with four queries each, norms: 4.5 us, of which a launch is more than half) and by HBM in large ones (4 prompts of 4096 tokens, 8
// heads, four queries each, 0.4 GB in and out: 92 us, into 4 bits 83).
template <bool FP4>
__global__ __launch_bounds__(256) void rotate_append_kernel(const CacheView C, const Rotation R, const RotateAppend S) {
  __shared__ uint4 exchange[FP4 ? 16 : 1][16];
  const int row = threadIdx.x >> 4, lane = threadIdx.x & 15, mine = row % S.head_rows;
  const unsigned block = blockIdx.x / (unsigned)S.parts;
  const int part = (int)(blockIdx.x - block * (unsigned)S.parts);
  const unsigned g = block * (unsigned)(16 / S.head_rows) + (unsigned)(row / S.head_rows);
  const bool real = g < (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads;
  const HeadOf w = head_of(C, real ? g : 0u);
  const HeadPlace hp = head_place(C, w);
  const int n = real ? tokens_new(S.new_tokens, w.b, S.tokens) : 0, count = held(C, w.b, w.l, w.h);
  const int seen = C.seen[count_at(C, w.b, w.l, w.h)];
  const RowPieces p = row_pieces(R, lane);
  const bool turned = lane < R.turned;
  double freqs[4];
  turn_freqs(R, lane, freqs);
  Weights qw, kw;
  if (R.q_norm != nullptr && S.group > 0) load_weights(R.q_norm, w.l, p, qw);
  if (R.k_norm != nullptr) load_weights(R.k_norm, w.l, p, kw);
  const int from = part * S.part, to = n - from < S.part ? n : from + S.part;
  for (int t = from + mine / S.token_rows; t < to; t += S.head_rows / S.token_rows) {
    const int position = (int)((unsigned)seen + (unsigned)t);
    Turn turn;
    turn_of(R, freqs, position, turn);
    const long long src = w.b * S.stride_b + w.l * S.stride_l + t * S.stride_t + w.h * S.stride_h;
    const bool room = t < C.capacity - count;
    SlotPlace s{-1, 0};
    if (room) s = slot_place(C, hp, count + t);
    const bool there = room && page_there(C, s.page);
    for (int r = mine % S.token_rows; r < S.group + 2; r += S.token_rows) {
      if (r >= 2) {
        const int h = w.h * S.group + r - 2;
        float y[8];
        norm_row(load_raw(S.q + w.b * S.q_b + w.l * S.q_l + t * S.q_t + h * S.q_h, p), R.q_norm != nullptr, qw, R.eps, y);
        store_raw(S.q_out + w.b * S.qo_b + w.l * S.qo_l + t * S.qo_t + h * S.qo_h, p, turn_row(R, turn, turned, y));
        continue;
      }
      if (!there) continue;
      const long long dst = row_at(C, hp, s), at = state_at(C, hp, s);
      if (r == 0) {
        float y[8];
        norm_row(load_raw(S.k + src, p), R.k_norm != nullptr, kw, R.eps, y);
        const Raw z = turn_row(R, turn, turned, y);
        if (FP4) {                 // into the order of 8 channels a lane
          store_raw(reinterpret_cast<uint16_t *>(exchange[row]), p, z);
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
          const uint4 x = exchange[row][lane];
          uint32_t scales;
          reinterpret_cast<unsigned *>(C.k + dst)[lane] = fp4_encode_row(x, lane, scales);
          if (lane == 0) C.k_scales[at] = scales;
        } else {
          store_raw(C.k + dst, p, z);
        }
        if (lane == 0) {
          C.mass[at] = 0.f;
          C.positions[at] = position;
        }
      } else {
        const uint4 x = *reinterpret_cast<const uint4 *>(S.v + src + 8 * lane);
        if (FP4) {
          uint32_t scales;
          reinterpret_cast<unsigned *>(C.v + dst)[lane] = fp4_encode_row(x, lane, scales);
          if (lane == 0) C.v_scales[at] = scales;
        } else {
          *reinterpret_cast<uint4 *>(C.v + dst + 8 * lane) = x;
        }
      }
    }
  }
  if (S.parts > 1) return;         // another launch moves the counts on
  __syncthreads();                 // every wave has read them
  if (mine == 0 && lane == 0 && n > 0) append_count(C, w, count, seen, n);
}
__global__ __launch_bounds__(256) void rotate_counts_kernel(const CacheView C, const int32_t *new_tokens, int tokens) {
  const unsigned g = blockIdx.x * 256u + threadIdx.x;
  if (g >= (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads) return;
  const HeadOf w = head_of(C, g);
  const int n = tokens_new(new_tokens, w.b, tokens);
  if (n > 0) append_count(C, w, held(C, w.b, w.l, w.h), C.seen[count_at(C, w.b, w.l, w.h)], n);
}

// ------------------------------------------------------------------------------------------ calls
static bool misaligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Strides of bf16 rows that 8-byte pieces (and 16-byte ones of values) are read by.
static int strides_check(long long b, long long l, long long t, long long h) {
  if (b < 0 || l < 0 || t < 0 || h < 0) return COMPACTOR_EINVAL;
  return (b | l | t | h) & 7 ? COMPACTOR_EALIGN : COMPACTOR_OK;
}

static int rotation_of(const compactor_rotation_t *r, Rotation *R) {
  if (!r || !r->freqs) return COMPACTOR_EINVAL;
  if (r->rotary_dim < 8 || r->rotary_dim > D || r->rotary_dim % 8) return COMPACTOR_EUNSUPPORTED;
  if ((r->q_norm || r->k_norm) && !(r->eps >= 0x1p-100f && r->eps <= 3e38f)) return COMPACTOR_EINVAL;
  if (misaligned(r->freqs, 8) || misaligned(r->q_norm, 16) || misaligned(r->k_norm, 16)) return COMPACTOR_EALIGN;
  *R = Rotation{r->freqs, r->q_norm, r->k_norm, r->rotary_dim / 8, r->interleaved ? 1 : 0, r->eps};
  return COMPACTOR_OK;
}

static int append_rotated(const CacheView &C, const compactor_rotation_t *rotation, const compactor_cache_rows_t *rows,
                          const compactor_rotate_queries_t *queries, void *stream) {
  Rotation R;
  int rc = rotation_of(rotation, &R);
  if (rc) return rc;
  if (!rows || !rows->k || !rows->v || rows->tokens < 1) return COMPACTOR_EINVAL;
  if ((rc = strides_check(rows->stride_b, rows->stride_l, rows->stride_t, rows->stride_h)) != 0) return rc;
  if (misaligned(rows->k, 16) || misaligned(rows->v, 16) || misaligned(rows->new_tokens, 4)) return COMPACTOR_EALIGN;
  RotateAppend S{};
  S.k = static_cast<const uint16_t *>(rows->k);
  S.v = static_cast<const uint16_t *>(rows->v);
  S.stride_b = rows->stride_b; S.stride_l = rows->stride_l;
  S.stride_t = rows->stride_t; S.stride_h = rows->stride_h;
  S.new_tokens = rows->new_tokens;
  S.tokens = rows->tokens;
  if (queries) {
    const compactor_rotate_queries_t &q = *queries;
    if (!q.q || !q.q_out || q.q_heads < C.kv_heads || q.q_heads % C.kv_heads || q.q_heads > HEADS_MOST) return COMPACTOR_EINVAL;
    if ((rc = strides_check(q.q_stride_b, q.q_stride_l, q.q_stride_t, q.q_stride_h)) != 0) return rc;
    if ((rc = strides_check(q.q_out_stride_b, q.q_out_stride_l, q.q_out_stride_t, q.q_out_stride_h)) != 0) return rc;
    if (misaligned(q.q, 16) || misaligned(q.q_out, 16)) return COMPACTOR_EALIGN;
    if (q.q == q.q_out && (q.q_stride_b != q.q_out_stride_b || q.q_stride_l != q.q_out_stride_l || q.q_stride_t != q.q_out_stride_t ||
                           q.q_stride_h != q.q_out_stride_h))
      return COMPACTOR_EINVAL;
    S.q = static_cast<const uint16_t *>(q.q);
    S.q_out = static_cast<uint16_t *>(q.q_out);
    S.q_b = q.q_stride_b; S.q_l = q.q_stride_l; S.q_t = q.q_stride_t; S.q_h = q.q_stride_h;
    S.qo_b = q.q_out_stride_b; S.qo_l = q.q_out_stride_l; S.qo_t = q.q_out_stride_t; S.qo_h = q.q_out_stride_h;
    S.group = q.q_heads / C.kv_heads;
  }
  // One token: a head's rows side by side, of as many heads as fit.  A few: two rows of lanes a token, eight tokens side by side; more: one, so that a turn is
  // found once (us of 4 prompts of 4096 tokens, 8 heads, 4 queries each, with 4, 2 and 1 rows: 168, 107 and 92; 16 of 8 tokens 6.9, 5.1 and 5.8).
  // Parts of a head are as long as leaves every unit 16 workgroups (4 prompts of 64: 7.4 us with 16 tokens a part, 10 with 32, 14 with 64; 64 of 64 22.6, 26.4, 23.4).
  S.head_rows = S.tokens > 1 ? 16 : S.group <= 2 ? 4 : S.group <= 6 ? 8 : 16;
  S.token_rows = S.tokens == 1 ? S.head_rows : S.tokens <= 8 ? 2 : 1;
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  auto parts_of = [&](int part) { return ((long long)S.tokens + part - 1) / part; };
  for (S.part = 64; S.part > 16 && heads * parts_of(S.part) < 4096;) S.part /= 2;
  S.parts = (int)parts_of(S.part);
  const long long per = 16 / S.head_rows, blocks = (heads + per - 1) / per * S.parts;
  if (!launchable(blocks, 256) || !launchable((heads + 255) / 256, 256)) return COMPACTOR_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(C.k_scales != nullptr ? rotate_append_kernel<true> : rotate_append_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st,
                     C, R, S);
  if (S.parts > 1) {
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    hipLaunchKernelGGL(rotate_counts_kernel, dim3((unsigned)((heads + 255) / 256)), dim3(256), 0, st, C, S.new_tokens, S.tokens);
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_rotate(const compactor_rotation_t *rotation, const compactor_rotate_rows_t *rows, void *stream) {
  Rotation R;
  int rc = rotation_of(rotation, &R);
  if (rc) return rc;
  if (!rows) return COMPACTOR_EINVAL;
  const compactor_rotate_rows_t &r = *rows;
  if (r.nreq < 1 || r.layers < 1 || r.tokens < 1 || r.q_heads < 0 || r.kv_heads < 0 || r.q_heads + (long long)r.kv_heads < 1) return COMPACTOR_EINVAL;
  if (r.q_heads > HEADS_MOST || r.kv_heads > HEADS_MOST) return COMPACTOR_EINVAL;
  if (!r.positions || r.position_stride_b < 0) return COMPACTOR_EINVAL;
  if (misaligned(r.positions, 4) || misaligned(r.new_tokens, 4)) return COMPACTOR_EALIGN;
  if (r.q_heads > 0) {
    if (!r.q || !r.q_out) return COMPACTOR_EINVAL;
    if ((rc = strides_check(r.q_stride_b, r.q_stride_l, r.q_stride_t, r.q_stride_h)) != 0) return rc;
    if ((rc = strides_check(r.q_out_stride_b, r.q_out_stride_l, r.q_out_stride_t, r.q_out_stride_h)) != 0) return rc;
    if (misaligned(r.q, 16) || misaligned(r.q_out, 16)) return COMPACTOR_EALIGN;
    if (r.q == r.q_out && (r.q_stride_b != r.q_out_stride_b || r.q_stride_l != r.q_out_stride_l || r.q_stride_t != r.q_out_stride_t ||
                           r.q_stride_h != r.q_out_stride_h))
      return COMPACTOR_EINVAL;
  }
  if (r.kv_heads > 0) {
    if (!r.k || !r.k_out || r.k_plain == r.k_out) return COMPACTOR_EINVAL;
    if ((rc = strides_check(r.k_stride_b, r.k_stride_l, r.k_stride_t, r.k_stride_h)) != 0) return rc;
    if ((rc = strides_check(r.k_out_stride_b, r.k_out_stride_l, r.k_out_stride_t, r.k_out_stride_h)) != 0) return rc;
    if (misaligned(r.k, 16) || misaligned(r.k_out, 16)) return COMPACTOR_EALIGN;
    if (r.k == r.k_out && (r.k_stride_b != r.k_out_stride_b || r.k_stride_l != r.k_out_stride_l || r.k_stride_t != r.k_out_stride_t ||
                           r.k_stride_h != r.k_out_stride_h))
      return COMPACTOR_EINVAL;
    if (r.k_plain) {
      if ((rc = strides_check(r.k_plain_stride_b, r.k_plain_stride_l, r.k_plain_stride_t, r.k_plain_stride_h)) != 0) return rc;
      if (misaligned(r.k_plain, 16)) return COMPACTOR_EALIGN;
      if (r.k == r.k_plain && (r.k_stride_b != r.k_plain_stride_b || r.k_stride_l != r.k_plain_stride_l || r.k_stride_t != r.k_plain_stride_t ||
                               r.k_stride_h != r.k_plain_stride_h))
        return COMPACTOR_EINVAL;
    }
  }
  if (r.q_heads > 0 && r.kv_heads > 0 && (r.q_out == r.k_out || r.q_out == r.k_plain || r.q_out == r.k || r.k_out == r.q || r.k_plain == r.q))
    return COMPACTOR_EINVAL;
  const long long tokens = (long long)r.nreq * r.layers * r.tokens;
  if ((long long)r.nreq * r.layers > 0x7fffffffll || tokens > 0x7fffffffll) return COMPACTOR_EINVAL;
  RotateRows S{static_cast<const uint16_t *>(r.q), static_cast<const uint16_t *>(r.k), static_cast<uint16_t *>(r.q_out),
               static_cast<uint16_t *>(r.k_out), static_cast<uint16_t *>(r.k_plain),
               r.q_stride_b, r.q_stride_l, r.q_stride_t, r.q_stride_h, r.k_stride_b, r.k_stride_l, r.k_stride_t, r.k_stride_h,
               r.q_out_stride_b, r.q_out_stride_l, r.q_out_stride_t, r.q_out_stride_h,
               r.k_out_stride_b, r.k_out_stride_l, r.k_out_stride_t, r.k_out_stride_h,
               r.k_plain_stride_b, r.k_plain_stride_l, r.k_plain_stride_t, r.k_plain_stride_h,
               r.positions, r.position_stride_b, r.new_tokens, r.layers, r.tokens, r.q_heads, r.kv_heads, 1, 0u};
  // Few tokens: their heads over as many waves as have one for every row of lanes, up to a wave a SIMD of the chip (512 tokens of 32 + 8 heads: 5.7 us, with
  // four waves a SIMD 6.3; 2000 of 128 + 8 24.8 and 31).
  const int most = (max(r.q_heads, r.kv_heads) + 3) / 4;
  while (S.parts < most && tokens * S.parts < 1024) S.parts *= 2;
  const long long units = tokens * S.parts;
  if (units > 0x7fffffffll || !launchable((units + 3) / 4, 256)) return COMPACTOR_EINVAL;
  S.units = (unsigned)units;
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(rotate_kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, static_cast<hipStream_t>(stream), R, S);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

int compactor_cache_append_rotated(const compactor_cache_t *cache, const compactor_rotation_t *rotation, const compactor_cache_rows_t *rows,
                                   const compactor_rotate_queries_t *queries, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_STATE, &C);
  return rc ? rc : append_rotated(C, rotation, rows, queries, stream);
}

int compactor_mx_append_rotated(const compactor_mx_cache_t *cache, const compactor_rotation_t *rotation, const compactor_cache_rows_t *rows,
                                const compactor_rotate_queries_t *queries, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_STATE, &C);
  return rc ? rc : append_rotated(C, rotation, rows, queries, stream);
}

#pragma GCC visibility pop
}  // extern "C"
