// E4M3 codes with one fp32 scale per block of 128: helpers shared by the quantisation kernels and the Linear-1 epilogues.
#pragma once
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace blk {

// amax / 448, 1 for an all-zero block; a true division, so that codes and scales are reproducible bit for bit.
__device__ __forceinline__ float scale_of(float amax) { return amax > 0.f ? __fdiv_rn(amax, 448.f) : 1.f; }

// Division of many values by one scale: quotient from the correctly rounded reciprocal, its remainder by one fused
// multiply-add, and the correction by another (Markstein's scheme), three instructions per value where a general division
// takes about ten.  The remainder is taken with its sign turned, q scale - v: so a negative zero keeps its sign (v - q scale
// would be +0 + -0 = +0 and turn it).
struct FastDivider {
  float scale, reciprocal;
  __device__ __forceinline__ float operator()(float v) const {
    const float q = v * reciprocal;
    return fmaf(fmaf(q, scale, -v), -reciprocal, q);
  }
};
// From 2^-90 to 2^100 the reciprocal is a normal number and the remainder of a quotient of at least 2^-12 (a quarter of the
// smallest code) exact: its last bit is worth 2^-35 2^-113 or more.  Other scales, infinite ones among them, take the general division.
struct GeneralDivider {
  float scale;
  __device__ __forceinline__ float operator()(float v) const { return __fdiv_rn(v, scale); }
};
__device__ __forceinline__ bool general_scale(float scale) { return !(scale >= 0x1p-90f && scale <= 0x1p100f); }

// Four values over one scale -> four E4M3 codes in a word (lowest byte first), nearest-even, saturating; NaN stays NaN.
template <typename Divider>
__device__ __forceinline__ uint32_t pack4(const float* v, const Divider& by) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(by(v[0]), by(v[1])), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(by(v[2]), by(v[3])), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// N values over one scale -> N / 4 words.
template <int N>
__device__ __forceinline__ void pack(const float (&v)[N], float scale, uint32_t (&w)[N / 4]) {
  if (general_scale(scale)) {
    const GeneralDivider by{scale};
#pragma unroll
      for (int j = 0; j < N / 4; ++j) w[j] = pack4(v + 4 * j, by);
  } else {
    const FastDivider by{scale, __frcp_rn(scale)};
#pragma unroll
    for (int j = 0; j < N / 4; ++j) w[j] = pack4(v + 4 * j, by);
  }
}

}  // namespace blk
