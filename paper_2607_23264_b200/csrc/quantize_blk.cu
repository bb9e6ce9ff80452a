// Quantisation in blocks of 128: bf16 -> E4M3 codes and fp32 scales.
//
// quantize_rows_blk    : 16 lanes per 1 x 128 block, eight values (16 bytes) per lane; the block maximum is taken on bf16
//                        pairs and four shuffles, every lane converts and stores its eight codes.  A warp takes two
//                        blocks of a row per step and up to four steps' loads are in flight.
// quantize_dispatch_blk: the same, and the codes and the scale go to the k rows of the expert-contiguous buffer instead
//                        of to one row: a token is read once, quantised once and written k times, with no quantised copy
//                        of the batch in between.
// quantize_weights_blk : a CTA per 128 x 128 block, 64 values per thread kept in registers between the maximum and the
//                        conversion, so the block is read once.
//
// Each value is read and each code written once: 3 bytes a value, bound by HBM where the tensor is large.
// 8 x 14336 x 4096 weights: 244 us (1.41 GB, 5.8 TB/s).  1001 x 7168 rows: 6.3 us in a graph replay (22 MB; a launch
// is half of it).  Four values are converted with three multiply-adds each instead of a division (blk_quant.cuh): with
// the division the weights took 394 us, bound by instructions.
#include <cuda_bf16.h>

#include "blk_quant.cuh"
#include "moe_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kSteps = 4;                 // steps of two blocks whose loads are in flight together

__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// The larger magnitude per half of two pairs of bf16 (a NaN gives way to a number).
__device__ __forceinline__ __nv_bfloat162 amax_pair(__nv_bfloat162 m, uint32_t w) {
  return __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w)));
}
__device__ __forceinline__ __nv_bfloat162 amax8(__nv_bfloat162 m, const uint4& q) {
  return amax_pair(amax_pair(amax_pair(amax_pair(m, q.x), q.y), q.z), q.w);
}
__device__ __forceinline__ float larger_half(__nv_bfloat162 m) { return fmaxf(__low2float(m), __high2float(m)); }

// One row (or `steps` of it from block b0) by one warp; write(v, codes) takes vector v of the row, scale(b, s) block b.
template <typename Write, typename Scale>
__device__ __forceinline__ void quantize_span(const uint4* __restrict__ src, int vec_per_row, int b0, int b1, int lane,
                                              Write write, Scale scale) {
  const int sub = lane & 15, odd = lane >> 4;
  for (int b = b0; b < b1; b += 2 * kSteps) {
    uint4 q[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int blk_at = b + 2 * u + odd, v = blk_at * 16 + sub;
      q[u] = make_uint4(0u, 0u, 0u, 0u);
      if (blk_at < b1 && v < vec_per_row) q[u] = __ldg(src + v);
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      if (b + 2 * u >= b1) break;                        // (uniform: the shuffles need every lane)
      const int blk_at = b + 2 * u + odd, v = blk_at * 16 + sub;
      float amax = larger_half(amax8(__nv_bfloat162(__float2bfloat16_rn(0.f), __float2bfloat16_rn(0.f)), q[u]));
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
      const float sc = blk::scale_of(amax);
      float f[8];
      unpack8(q[u], f);
      uint32_t w[2];
      blk::pack(f, sc, w);
      write(v, blk_at < b1 && v < vec_per_row, make_uint2(w[0], w[1]));
      if (blk_at < b1) scale(blk_at, sub, sc);
    }
  }
}

// Item = one row x `span` blocks (a multiple of 2 * kSteps, or the whole row).
__global__ void __launch_bounds__(kThreads)
quantize_rows_blk(const uint4* __restrict__ in, int rows, int vec_per_row, int blocks_per_row, int span, int spans,
                  uint2* __restrict__ codes, float* __restrict__ scales) {
  const int lane = threadIdx.x & 31;
  const int item = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int row = item / spans;
  if (row >= rows) return;
  const int b0 = (item - row * spans) * span, b1 = min(b0 + span, blocks_per_row);
  const size_t at = static_cast<size_t>(row) * vec_per_row;
  quantize_span(
      in + at, vec_per_row, b0, b1, lane,
      [&](int v, bool mine, const uint2& w) {
        if (mine) codes[at + v] = w;
      },
      [&](int b, int sub, float sc) {
        if (sub == 0) scales[static_cast<size_t>(b) * rows + row] = sc;
      });
}

__global__ void __launch_bounds__(kThreads)
quantize_dispatch_blk(const uint4* __restrict__ x, const int32_t* __restrict__ inv_perm, int T, int k, int vec_per_row,
                      int blocks_per_row, int span, int spans, uint2* __restrict__ xq_perm, float* __restrict__ sx_perm) {
  const int lane = threadIdx.x & 31;
  const int item = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int t = item / spans;
  if (t >= T) return;
  const int b0 = (item - t * spans) * span, b1 = min(b0 + span, blocks_per_row);
  const int my_row = lane < k ? __ldg(inv_perm + static_cast<size_t>(t) * k + lane) : 0;
  const size_t R = static_cast<size_t>(T) * k;
  quantize_span(
      x + static_cast<size_t>(t) * vec_per_row, vec_per_row, b0, b1, lane,
      [&](int v, bool mine, const uint2& w) {
        for (int j = 0; j < k; ++j) {
          const int row = __shfl_sync(0xFFFFFFFFu, my_row, j);
          if (mine) xq_perm[static_cast<size_t>(row) * vec_per_row + v] = w;
        }
      },
      // the k scales of a block by k of its 16 lanes (k <= 32: two each at most)
      [&](int b, int sub, float sc) {
        for (int j = sub; j < k; j += 16)
          sx_perm[static_cast<size_t>(b) * R + __ldg(inv_perm + static_cast<size_t>(t) * k + j)] = sc;
      });
}

__global__ void __launch_bounds__(kThreads)
quantize_weights_blk(const uint4* __restrict__ in, int rows, int vec_per_row, int row_blocks, int col_blocks,
                     uint2* __restrict__ codes, float* __restrict__ scales) {
  __shared__ float s_part[kThreads / 32];
  const int tid = threadIdx.x;
  const int cb = static_cast<int>(blockIdx.x % static_cast<unsigned>(col_blocks));
  const unsigned rest = blockIdx.x / static_cast<unsigned>(col_blocks);
  const int rb = static_cast<int>(rest % static_cast<unsigned>(row_blocks));
  const size_t mat = rest / static_cast<unsigned>(row_blocks);
  const int v = cb * 16 + (tid & 15), r0 = rb * 128 + (tid >> 4);
  const size_t at = (mat * rows + r0) * vec_per_row + v;     // this thread's vectors: every sixteenth row
  const size_t pitch = static_cast<size_t>(16) * vec_per_row;
  uint4 q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    q[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r0 + 16 * i < rows && v < vec_per_row) q[i] = __ldg(in + at + i * pitch);
  }
  __nv_bfloat162 m(__float2bfloat16_rn(0.f), __float2bfloat16_rn(0.f));
#pragma unroll
  for (int i = 0; i < 8; ++i) m = amax8(m, q[i]);
  float amax = larger_half(m);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
  if ((tid & 31) == 0) s_part[tid >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) amax = fmaxf(amax, s_part[i]);
  const float sc = blk::scale_of(amax);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (r0 + 16 * i < rows && v < vec_per_row) {
      float f[8];
      unpack8(q[i], f);
      uint32_t w[2];
      blk::pack(f, sc, w);
      codes[at + i * pitch] = make_uint2(w[0], w[1]);
    }
  }
  if (tid == 0) scales[(mat * row_blocks + rb) * col_blocks + cb] = sc;
}

// Blocks per item: whole rows, cut into spans while that leaves fewer than eight warps per scheduler.
int span_of(const moe_ctx* ctx, long long rows, int blocks_per_row) {
  int span = blocks_per_row;
  while (span > 2 * kSteps && rows * ((blocks_per_row + span - 1) / span) < 32LL * ctx->num_sms)
    span = ((span + 1) / 2 + 2 * kSteps - 1) / (2 * kSteps) * (2 * kSteps);
  return span;
}

}  // namespace

namespace moe {

cudaError_t launch_quantize_rows_blk(moe_ctx* ctx, const void* in_bf16, long long rows, int cols, void* codes,
                                     float* scales, cudaStream_t stream) {
  if (rows == 0) return cudaSuccess;
  const int blocks_per_row = blocks_of(cols, 128);
  const int span = span_of(ctx, rows, blocks_per_row), spans = (blocks_per_row + span - 1) / span;
  const long long grid = (rows * spans + kThreads / 32 - 1) / (kThreads / 32);
  if (rows * spans > 0x7FFFFFFFLL - kThreads) return cudaErrorInvalidConfiguration;
  quantize_rows_blk<<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(
      static_cast<const uint4*>(in_bf16), static_cast<int>(rows), cols / 8, blocks_per_row, span, spans,
      static_cast<uint2*>(codes), scales);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

cudaError_t launch_quantize_dispatch_blk(moe_ctx* ctx, const void* x, const int32_t* inv_perm, void* xq_perm,
                                         float* sx_perm, cudaStream_t stream) {
  const moe_shape& s = ctx->shape;
  const int blocks_per_row = s.H / 128;
  const int span = span_of(ctx, s.T, blocks_per_row), spans = (blocks_per_row + span - 1) / span;
  const long long items = static_cast<long long>(s.T) * spans;
  if (items > 0x7FFFFFFFLL - kThreads) return cudaErrorInvalidConfiguration;
  quantize_dispatch_blk<<<static_cast<unsigned>((items + kThreads / 32 - 1) / (kThreads / 32)), kThreads, 0, stream>>>(
      static_cast<const uint4*>(x), inv_perm, s.T, s.k, s.H / 8, blocks_per_row, span, spans,
      static_cast<uint2*>(xq_perm), sx_perm);
  moe_mark(ctx, 4, stream);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

cudaError_t launch_quantize_weights_blk(moe_ctx* ctx, const void* in_bf16, long long mats, int rows, int cols,
                                        void* codes, float* scales, cudaStream_t stream) {
  const int rb = blocks_of(rows, 128), cb = blocks_of(cols, 128);
  const long long per_mat = static_cast<long long>(rb) * cb;
  if (per_mat > 0x7FFFFFFFLL / mats) return cudaErrorInvalidConfiguration;
  const long long grid = mats * per_mat;
  quantize_weights_blk<<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(
      static_cast<const uint4*>(in_bf16), rows, cols / 8, rb, cb, static_cast<uint2*>(codes), scales);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

}  // namespace moe
