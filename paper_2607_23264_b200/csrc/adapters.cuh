// What the kernels of the adapters share: arguments, t as two bf16 terms, and sums that the terms cannot form.
#pragma once
#include <cuda_bf16.h>

#include "moe_internal.h"

namespace moe {

struct AdapterParams {
  const __nv_bfloat16* x;
  const __nv_bfloat16* a;
  const __nv_bfloat16* b;
  const float* scale;
  const int32_t* offsets;
  const int32_t* adapter_of;
  const __nv_bfloat16* y_in;
  __nv_bfloat16* y_out;
  int32_t* status;
  long long rows;
  int N, K, rank, adapters, segments;
};

// 16 bytes into the shared memory of any CTA of the cluster.
__device__ __forceinline__ void st_cluster(uint32_t at, const uint4& v) {
  asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint32_t pair(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two values as two terms of bf16 each: v - hi is exact, so hi + lo keeps 16 bits.  hi stays finite: a value near fp32's end would
// round to an infinity, whose lo were one of the other sign (an infinite v: the largest bf16 and an infinity).
__device__ __forceinline__ void two_terms(float v0, float v1, uint32_t& hi, uint32_t& lo) {
  asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(v1), "f"(v0));
  lo = pair(v0 - low(hi), v1 - high(hi));
}

// Where b is infinite, hi b + lo b is NaN although t b is an infinity: 0 inf where t needs one term only, infinities of both signs
// where the terms differ in sign.  So sums that came out NaN are formed again from whole t.
// A NaN sum is packed as 0x7FFF, which as an integer lies above all other bf16: the largest of pairs shows one.
__device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b, uint32_t c) { return __vimax3_s16x2(a, b, c); }
__device__ __forceinline__ bool has_nan(uint32_t w) { return low(w) != low(w) || high(w) != high(w); }
__device__ __forceinline__ bool is_nan(uint16_t bits) { return (bits & 0x7FFF) > 0x7F80; }

// Long segments: tiles of 128 rows on the tensor cores.
moe_status launch_adapter_tiles(moe_ctx* ctx, const AdapterParams& p, cudaStream_t stream);
cudaError_t prepare_adapter_tiles(moe_ctx* ctx);

}  // namespace moe
