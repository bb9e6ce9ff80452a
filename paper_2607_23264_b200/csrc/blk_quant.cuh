// E4M3 codes with one fp32 scale per block of 128: helpers shared by the quantisation kernels and the Linear-1 epilogues.
#pragma once
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace blk {

// amax / 448, 1 for an all-zero block; a true division, so that codes and scales are reproducible bit for bit.
__device__ __forceinline__ float scale_of(float amax) { return amax > 0.f ? __fdiv_rn(amax, 448.f) : 1.f; }

// Division of many values by one scale.  Quotient from the correctly rounded reciprocal, its remainder by one fused
// multiply-add, and the correction by another (Markstein's scheme): three instructions per value where a general
// division takes about ten.  Scales so small that the reciprocal or the remainder leaves the normal range, and infinite
// ones, take the general division.
struct Divider {
  float scale, reciprocal;
  bool general;
  __device__ __forceinline__ explicit Divider(float s) {
    scale = s;
    reciprocal = __frcp_rn(s);
    general = !(s >= 7.9e-31f && s <= 1.2e30f);          // 2^-100 .. 2^100
  }
  __device__ __forceinline__ float operator()(float v) const {
    if (general) return __fdiv_rn(v, scale);
    const float q = v * reciprocal;
    return fmaf(fmaf(-q, scale, v), reciprocal, q);
  }
};

// Four values over one scale -> four E4M3 codes in a word (lowest byte first), nearest-even, saturating; NaN stays NaN.
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, const Divider& by) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(by(a), by(b)), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(by(c), by(d)), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

}  // namespace blk
