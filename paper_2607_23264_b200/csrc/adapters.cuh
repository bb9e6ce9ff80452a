// What the kernels of the adapters share: arguments, and the adapter of a row.
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

// Long segments: tiles of 128 rows on the tensor cores.
moe_status launch_adapter_tiles(moe_ctx* ctx, const AdapterParams& p, cudaStream_t stream);
cudaError_t prepare_adapter_tiles(moe_ctx* ctx);

}  // namespace moe
