// E4M3 codes with one fp32 scale per block of 128: helpers shared by the quantisation kernels and the Linear-1 epilogue.
#pragma once
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace blk {

// amax / 448, 1 for an all-zero block; a true division, so that codes and scales are reproducible bit for bit.
__device__ __forceinline__ float scale_of(float amax) { return amax > 0.f ? __fdiv_rn(amax, 448.f) : 1.f; }

// Four values over one scale -> four E4M3 codes in a word (lowest byte first), nearest-even, saturating; NaN stays NaN.
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, float scale) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(a, scale), __fdiv_rn(b, scale)), __NV_SATFINITE,
                                               __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(c, scale), __fdiv_rn(d, scale)), __NV_SATFINITE,
                                               __NV_E4M3);
  return lo | (hi << 16);
}

}  // namespace blk
