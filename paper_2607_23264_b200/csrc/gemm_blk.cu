// Grouped product of E4M3 rows and weights with fp32 scales per block of 128, and the two expert GEMMs on it.
//
// One thread per output column, 16 rows per CTA: per block of 128 along K the rows' codes are widened into shared
// memory, each thread walks its weight row's 128 codes and keeps one fp32 partial sum per row, which is then scaled
// into the running sum.  Linear-1 carries two such sums (gate, up) and quantises its 128 columns of h in the epilogue.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "blk_quant.cuh"
#include "ffn_math.cuh"
#include "moe_internal.h"

namespace {

constexpr int kCols = 128;   // output columns (threads) per CTA
constexpr int kRows = 16;    // rows per CTA

struct BlkParams {
  const unsigned char* a;    // [rows, K]
  const float* sa;           // [kb][rows]
  const int32_t* offsets;    // [groups + 1] or null
  const unsigned char* b0;   // [groups, N, K]
  const unsigned char* b1;   // gated: the up matrix
  const float* sb0;          // [groups][nb][kb]
  const float* sb1;
  __nv_bfloat16* y;          // [rows, N]
  unsigned char* hq;         // gated: [rows, N]
  float* sh;                 // gated: [N/128][rows]
  float* h_dbg;
  long long rows;
  int N, K, groups;
};

__device__ __forceinline__ float fp8_value(unsigned char c) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(c, __NV_E4M3)));
}

template <bool kGated>
__global__ void __launch_bounds__(kCols)
gemm_blk_kernel(const BlkParams p) {
  __shared__ float s_a[kRows][128];
  __shared__ float s_sa[kRows];
  __shared__ float s_part[kCols / 32];
  __shared__ long long s_row0, s_end;
  __shared__ int s_group;
  const int tid = threadIdx.x;
  if (tid == 0) {
    s_group = -1;
    long long tile = blockIdx.y;
    for (int g = 0; g < p.groups; ++g) {
      long long lo = p.offsets ? p.offsets[g] : 0, hi = p.offsets ? p.offsets[g + 1] : p.rows;
      lo = lo < 0 ? 0 : lo;
      hi = hi > p.rows ? p.rows : hi;
      const long long n = hi > lo ? (hi - lo + kRows - 1) / kRows : 0;
      if (tile < n) {
        s_group = g;
        s_row0 = lo + tile * kRows;
        s_end = hi;
        break;
      }
      tile -= n;
    }
  }
  __syncthreads();
  if (s_group < 0) return;
  const int g = s_group, n = blockIdx.x * kCols + tid;
  const long long row0 = s_row0;
  const int live = static_cast<int>(min(static_cast<long long>(kRows), s_end - row0));
  const int kb_count = (p.K + 127) / 128, nb_count = (p.N + 127) / 128;
  const bool col_ok = n < p.N;
  float acc0[kRows], acc1[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) acc0[r] = acc1[r] = 0.f;
  for (int kb = 0; kb < kb_count; ++kb) {
    const int kn = min(128, p.K - kb * 128);
    __syncthreads();
    for (int r = 0; r < kRows; ++r)
      s_a[r][tid] = (r < live && tid < kn) ? fp8_value(p.a[(row0 + r) * p.K + kb * 128 + tid]) : 0.f;
    if (tid < kRows) s_sa[tid] = tid < live ? p.sa[static_cast<size_t>(kb) * p.rows + row0 + tid] : 0.f;
    __syncthreads();
    if (!col_ok) continue;
    const size_t w_at = (static_cast<size_t>(g) * p.N + n) * p.K + kb * 128;
    const size_t s_at = (static_cast<size_t>(g) * nb_count + blockIdx.x) * kb_count + kb;
    float part0[kRows], part1[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) part0[r] = part1[r] = 0.f;
    for (int c = 0; c < kn; ++c) {
      const float w0 = fp8_value(p.b0[w_at + c]);
      const float w1 = kGated ? fp8_value(p.b1[w_at + c]) : 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        part0[r] = fmaf(s_a[r][c], w0, part0[r]);
        if (kGated) part1[r] = fmaf(s_a[r][c], w1, part1[r]);
      }
    }
    const float sb0 = p.sb0[s_at], sb1 = kGated ? p.sb1[s_at] : 0.f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      acc0[r] = fmaf(part0[r], s_sa[r] * sb0, acc0[r]);
      if (kGated) acc1[r] = fmaf(part1[r], s_sa[r] * sb1, acc1[r]);
    }
  }
  if constexpr (!kGated) {
    if (col_ok)
      for (int r = 0; r < live; ++r) p.y[(row0 + r) * p.N + n] = __float2bfloat16_rn(acc0[r]);
  } else {
    for (int r = 0; r < live; ++r) {
      const float h = acc0[r] / (1.f + expf(-acc0[r])) * acc1[r];
      float amax = fabsf(h);
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
      if ((tid & 31) == 0) s_part[tid >> 5] = amax;
      __syncthreads();
      amax = fmaxf(fmaxf(s_part[0], s_part[1]), fmaxf(s_part[2], s_part[3]));
      __syncthreads();
      const float sc = blk::scale_of(amax);
      p.hq[(row0 + r) * p.N + n] =
          static_cast<unsigned char>(__nv_cvt_float_to_fp8(__fdiv_rn(h, sc), __NV_SATFINITE, __NV_E4M3));
      if (tid == 0) p.sh[static_cast<size_t>(blockIdx.x) * p.rows + row0 + r] = sc;
      if (p.h_dbg) p.h_dbg[(row0 + r) * p.N + n] = h;
    }
  }
}

dim3 grid_of(const BlkParams& p) {
  return dim3((p.N + kCols - 1) / kCols, static_cast<unsigned>(p.rows / kRows + p.groups));
}

}  // namespace

namespace moe {

moe_status launch_gemm_blk(moe_ctx* ctx, const moe_gemm_blk_args* a, cudaStream_t stream) {
  BlkParams p{};
  p.a = static_cast<const unsigned char*>(a->a);
  p.sa = a->sa;
  p.offsets = a->offsets;
  p.b0 = static_cast<const unsigned char*>(a->b);
  p.sb0 = a->sb;
  p.y = static_cast<__nv_bfloat16*>(a->y);
  p.rows = a->rows;
  p.N = a->N;
  p.K = a->K;
  p.groups = a->groups;
  gemm_blk_kernel<false><<<grid_of(p), kCols, 0, stream>>>(p);
  ctx->last_launches += 1;
  return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

moe_status launch_expert_ffn_blk(moe_ctx* ctx, const moe_blk_ffn_args* a, cudaStream_t stream) {
  const moe_shape& s = ctx->shape;
  BlkParams p{};
  p.a = static_cast<const unsigned char*>(a->xq_perm);
  p.sa = a->sx_perm;
  p.offsets = a->offsets;
  p.b0 = static_cast<const unsigned char*>(a->wq_gate);
  p.b1 = static_cast<const unsigned char*>(a->wq_up);
  p.sb0 = a->s_gate;
  p.sb1 = a->s_up;
  p.hq = static_cast<unsigned char*>(a->hq_ws);
  p.sh = a->sh_ws;
  p.h_dbg = a->h_fp32_debug;
  p.rows = static_cast<long long>(s.T) * s.k;
  p.N = s.F;
  p.K = s.H;
  p.groups = s.E;
  gemm_blk_kernel<true><<<grid_of(p), kCols, 0, stream>>>(p);
  moe_mark(ctx, 5, stream);
  p.a = static_cast<const unsigned char*>(a->hq_ws);
  p.sa = a->sh_ws;
  p.b0 = static_cast<const unsigned char*>(a->wq_down);
  p.sb0 = a->s_down;
  p.y = static_cast<__nv_bfloat16*>(a->y_perm);
  p.N = s.H;
  p.K = s.F;
  gemm_blk_kernel<false><<<grid_of(p), kCols, 0, stream>>>(p);
  moe_mark(ctx, 6, stream);
  ctx->last_launches += 2;
  return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // namespace moe
