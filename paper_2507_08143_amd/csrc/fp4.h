// Numbers of 4 bits: E2M1 codes, eight to a 32-bit word, and E8M0 scales, one for 32 channels (see compactor_mx_cache_t).  gfx950
// converts both ways itself, two at a time and with the scale, at the rate of any other vector instruction; decoding is exact in bf16.
#pragma once

#include "cache.h"

namespace cmp {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr unsigned FP4_LEAST = 2, FP4_MOST = 252;      // scale bytes: all values are normal bf16 numbers
constexpr unsigned FP4_NAN = 255;

// The scale of group g of a row's four, as the conversions take it.
__device__ __forceinline__ float fp4_scale(unsigned scales, int g) { return __uint_as_float((scales >> (8 * g) & 0xffu) << 23); }

// Two channels of byte `at` of a word in bf16.
template <int at>
__device__ __forceinline__ unsigned fp4_pair(unsigned word, float scale) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, at);
  unsigned u;
  __builtin_memcpy(&u, &x, 4);
  return u;
}
__device__ __forceinline__ uint4 fp4_decode(unsigned word, float scale) {
  return make_uint4(fp4_pair<0>(word, scale), fp4_pair<1>(word, scale), fp4_pair<2>(word, scale), fp4_pair<3>(word, scale));
}

// The scale byte of a group whose largest magnitude has these bits in bf16: 2^(k - 2) for m 2^k, one more from m = 1.75 on, where 7 lies.
__device__ __forceinline__ unsigned fp4_scale_byte(unsigned largest) {
  if (largest >= 0x7f80u) return FP4_NAN;
  const int s = (int)((largest + 0x20u) >> 7) - 2;
  return (unsigned)min(max(s, (int)FP4_LEAST), (int)FP4_MOST);
}
// Eight channels of bf16 to a word; a group that is NaN has codes 0.
__device__ __forceinline__ unsigned fp4_encode(const uint4 &x, unsigned byte) {
  const float scale = __uint_as_float(byte << 23);
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
  bf16x2 p[4];
  __builtin_memcpy(p, w, 16);
  unsigned u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, p[0], scale, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, p[1], scale, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, p[2], scale, 2);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, p[3], scale, 3);
  return byte == FP4_NAN ? 0u : u;
}

// A row by 16 lanes (of one DPP row), 8 channels a lane; four lanes share a group.  -> the lane's word; scales: all four, in every lane
__device__ __forceinline__ unsigned fp4_encode_row(const uint4 &x, int lane, uint32_t &scales) {
  unsigned top = 0;
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
  top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, false));       // the neighbour's, the other pair's
  top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, false));
  const unsigned byte = fp4_scale_byte(top);
  scales = byte << (8 * (lane >> 2));
  scales |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)scales, 0x124, 0xf, 0xf, false);         // of the lanes 4 and 8 further round the row
  scales |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)scales, 0x128, 0xf, 0xf, false);
  return fp4_encode(x, byte);
}

}  // namespace cmp
