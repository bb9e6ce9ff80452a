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
  float* t;                               // [splits][rows][rank]
  int32_t* status;
  long long rows;
  int N, K, rank, adapters, segments, splits;
};

// The adapter of a row, -1 without one.  `offsets` and `adapter_of` are p's or copies of them.
__device__ __forceinline__ int adapter_of_row(const AdapterParams& p, const int32_t* offsets, const int32_t* adapter_of,
                                              long long row, bool report) {
  if (row >= p.rows) return -1;
  int seg = static_cast<int>(row);
  if (offsets != nullptr) {
    int lo = -1, hi = p.segments;                          // the last segment that begins at or before the row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid] <= row) lo = mid;
      else hi = mid;
    }
    if (lo < 0 || row >= offsets[lo + 1]) return -1;
    seg = lo;
  }
  const int id = adapter_of[seg];
  if (id >= p.adapters) {
    if (report) {
      atomicCAS(&p.status[0], 0, MOE_ERR_BAD_ROUTING);
      atomicCAS(&p.status[1], 0, seg);
    }
    return -1;
  }
  return id < 0 ? -1 : id;
}

// Long segments: tiles of 128 rows on the tensor cores.
moe_status launch_adapter_tiles(moe_ctx* ctx, const AdapterParams& p, cudaStream_t stream);

}  // namespace moe
