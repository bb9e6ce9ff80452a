// Quantisation in blocks of 128: bf16 -> E4M3 codes and fp32 scales.
//
// quantize_rows_blk    : 16 lanes per 1 x 128 block, eight values (16 bytes) per lane; the block maximum is four
//                        shuffles, every lane converts and stores its eight codes.
// quantize_weights_blk : a CTA per 128 x 128 block, 64 values per thread kept in registers between the maximum and the
//                        conversion, so the block is read once.
#include <cuda_bf16.h>

#include "blk_quant.cuh"
#include "moe_internal.h"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&q);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __bfloat1622float2(p[i]);
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ float amax8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}

// vec_per_row = cols / 8; the last block of a row may be short.
__global__ void __launch_bounds__(kThreads)
quantize_rows_blk(const uint4* __restrict__ in, long long rows, int vec_per_row, int blocks_per_row,
                  uint2* __restrict__ codes, float* __restrict__ scales) {
  const int sub = threadIdx.x & 15;
  const long long total = rows * blocks_per_row;
  const long long step = static_cast<long long>(gridDim.x) * (kThreads / 16);
  // the two halves of a warp run the same number of rounds: the shuffles need every lane
  const long long first = (static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x) / 32 * 2;
  for (long long g0 = first; g0 < total; g0 += step) {
    const long long g = g0 + ((threadIdx.x >> 4) & 1);
    const bool live = g < total;
    const long long row = live ? g / blocks_per_row : 0;
    const int b = live ? static_cast<int>(g - row * blocks_per_row) : 0;
    const int v = b * 16 + sub;
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const bool mine = live && v < vec_per_row;
    if (mine) unpack8(__ldg(in + row * vec_per_row + v), f);
    float amax = amax8(f);
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
    const float sc = blk::scale_of(amax);
    const blk::Divider by(sc);
    if (mine)
      codes[row * vec_per_row + v] =
          make_uint2(blk::pack4(f[0], f[1], f[2], f[3], by), blk::pack4(f[4], f[5], f[6], f[7], by));
    if (live && sub == 0) scales[static_cast<size_t>(b) * rows + row] = sc;
  }
}

__global__ void __launch_bounds__(kThreads)
quantize_weights_blk(const uint4* __restrict__ in, int rows, int vec_per_row, int row_blocks, int col_blocks,
                     uint2* __restrict__ codes, float* __restrict__ scales) {
  __shared__ float s_part[kThreads / 32];
  const int tid = threadIdx.x;
  const long long blk_id = blockIdx.x;
  const int cb = static_cast<int>(blk_id % col_blocks);
  const int rb = static_cast<int>((blk_id / col_blocks) % row_blocks);
  const long long mat = blk_id / (static_cast<long long>(col_blocks) * row_blocks);
  const int v = cb * 16 + (tid & 15);
  uint4 q[8];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rb * 128 + i * 16 + (tid >> 4);
    q[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r < rows && v < vec_per_row) q[i] = __ldg(in + (mat * rows + r) * vec_per_row + v);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float f[8];
    unpack8(q[i], f);
    amax = fmaxf(amax, amax8(f));
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
  if ((tid & 31) == 0) s_part[tid >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) amax = fmaxf(amax, s_part[i]);
  const float sc = blk::scale_of(amax);
  const blk::Divider by(sc);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rb * 128 + i * 16 + (tid >> 4);
    if (r < rows && v < vec_per_row) {
      float f[8];
      unpack8(q[i], f);
      codes[(mat * rows + r) * vec_per_row + v] =
          make_uint2(blk::pack4(f[0], f[1], f[2], f[3], by), blk::pack4(f[4], f[5], f[6], f[7], by));
    }
  }
  if (tid == 0) scales[(mat * row_blocks + rb) * col_blocks + cb] = sc;
}

}  // namespace

namespace moe {

cudaError_t launch_quantize_rows_blk(moe_ctx* ctx, const void* in_bf16, long long rows, int cols, void* codes,
                                     float* scales, cudaStream_t stream) {
  if (rows == 0) return cudaSuccess;
  const int blocks_per_row = (cols + 127) / 128;
  const long long total = rows * blocks_per_row;
  long long grid = (total + kThreads / 16 - 1) / (kThreads / 16);
  const long long cap = static_cast<long long>(ctx->num_sms) * 32;
  if (grid > cap) grid = cap;
  quantize_rows_blk<<<static_cast<int>(grid), kThreads, 0, stream>>>(static_cast<const uint4*>(in_bf16), rows, cols / 8,
                                                                    blocks_per_row, static_cast<uint2*>(codes), scales);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

cudaError_t launch_quantize_weights_blk(moe_ctx* ctx, const void* in_bf16, long long mats, int rows, int cols,
                                        void* codes, float* scales, cudaStream_t stream) {
  const int rb = (rows + 127) / 128, cb = (cols + 127) / 128;
  const long long grid = mats * rb * cb;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
  quantize_weights_blk<<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(
      static_cast<const uint4*>(in_bf16), rows, cols / 8, rb, cb, static_cast<uint2*>(codes), scales);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

}  // namespace moe
