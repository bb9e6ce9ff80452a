// Residual addition and RMS norm with an output in bf16, in 8 bits with scales, or both; and the norm's gradients.
//
// add_rms_norm  : kWarps warps per row, the row in registers (kVecs vectors of eight values per lane) from its one read to
//                 its last write.  s = bf16(x + residual): the fp32 sum of two bf16 numbers is exact, or so near the larger
//                 one that rounding it again gives that one, so s has one rounding.  The statistics are sums over s as
//                 stored: the gradient then sees the same function, from the same tensor.
// norm_backward : the same ownership of a row, persistent over rows, so that a lane's columns stay its own and the gain's
//                 gradient is summed in registers; one partial row per CTA, summed by norm_gain_sum in a fixed order.
#include <cuda_bf16.h>

#include "blk_quant.cuh"
#include "moe_internal.h"
#include "mx_quant.cuh"
#include "route_scored.cuh"

namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kBlock = 256;               // threads of a CTA, unless one row takes more

struct NormParams {
  const uint4* x;
  const uint4* residual;
  const void* gain;
  uint4* sum;
  uint4* out;
  uint2* codes;
  void* scales;
  long long rows;
  int vecs, cols;                         // vectors and values of a row
  float eps, gain_offset;
  int gain_fp32, form;
};

struct NormGradParams {
  const uint4* s;
  const void* gain;
  const uint4* d_out;
  const uint4* d_sum;
  uint4* d_x;
  float* partial;                         // [CTAs][cols], or null
  long long rows;
  int vecs, cols;
  float eps, gain_offset;
  int gain_fp32;
};

__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}
__device__ __forceinline__ void load_gain(const void* gain, int fp32, float offset, int v, float (&g)[8]) {
  if (fp32) {
    const float4 a = __ldg(static_cast<const float4*>(gain) + 2 * v), b = __ldg(static_cast<const float4*>(gain) + 2 * v + 1);
    g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w;
    g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
  } else {
    unpack8(__ldg(static_cast<const uint4*>(gain) + v), g);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] += offset;
}

// The warps of one row meet (named barriers: a CTA's last rows may be missing).
template <int kWarps>
__device__ __forceinline__ void row_sync(int group) {
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * kWarps) : "memory");
}
// Sum (or maximum) over the row's warps in a fixed order.  `part` holds kWarps floats per row of the CTA and may be written
// again once every warp of the row has met after the reads.
template <int kWarps>
__device__ __forceinline__ float row_sum(float v, float* part, int group, int warp, int lane) {
  v = moe::warp_sum(v);
  if constexpr (kWarps > 1) {
    if (lane == 0) part[warp] = v;
    row_sync<kWarps>(group);
    v = moe::warp_sum(lane < kWarps ? part[lane] : 0.f);
  }
  return v;
}
template <int kWarps>
__device__ __forceinline__ float row_max(float v, float* part, int group, int warp, int lane) {
  v = moe::warp_max(v);
  if constexpr (kWarps > 1) {
    if (lane == 0) part[warp] = v;
    row_sync<kWarps>(group);
    v = moe::warp_max(lane < kWarps ? part[lane] : 0.f);
  }
  return v;
}

__device__ __forceinline__ float amax8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}
// 1 / sqrt(mean + eps), correctly rounded.
__device__ __forceinline__ float rstd_of(float sum_of_squares, int cols, float eps) {
  return __frsqrt_rn(__fdiv_rn(sum_of_squares, static_cast<float>(cols)) + eps);
}

template <int kWarps, int kVecs>
__global__ void __launch_bounds__(kWarps * 32 > kBlock ? kWarps * 32 : kBlock)
add_rms_norm(const NormParams p) {
  constexpr int kGroups = kWarps * 32 >= kBlock ? 1 : kBlock / (kWarps * 32);
  constexpr int kLanes = kWarps * 32;
  __shared__ float s_part[2][kGroups * kWarps];
  const int lane = threadIdx.x & 31, group = threadIdx.x / kLanes, tid = threadIdx.x % kLanes, warp = tid >> 5;
  const long long row = static_cast<long long>(blockIdx.x) * kGroups + group;
  if (row >= p.rows) return;                               // (all warps of a row alike)
  const size_t at = static_cast<size_t>(row) * p.vecs;

  uint4 q[kVecs];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v = tid + i * kLanes;
    q[i] = make_uint4(0u, 0u, 0u, 0u);
    if (v < p.vecs) q[i] = p.x[at + v];
  }
  if (p.residual != nullptr) {
    uint4 r[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kLanes;
      r[i] = make_uint4(0u, 0u, 0u, 0u);
      if (v < p.vecs) r[i] = p.residual[at + v];
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float a[8], b[8];
      unpack8(q[i], a);
      unpack8(r[i], b);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] += b[j];
      q[i] = pack8(a);
    }
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    float a[8];
    unpack8(q[i], a);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(a[j], a[j], ss);
    const int v = tid + i * kLanes;
    if (p.sum != nullptr && v < p.vecs) p.sum[at + v] = q[i];
  }
  ss = row_sum<kWarps>(ss, s_part[0] + group * kWarps, group, warp, lane);
  const float rstd = rstd_of(ss, p.cols, p.eps);

  float row_scale = 1.f;
  if (p.form == MOE_FORM_ROWS) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kLanes;
      if (v < p.vecs) {
        float a[8], g[8];
        unpack8(q[i], a);
        load_gain(p.gain, p.gain_fp32, p.gain_offset, v, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = a[j] * rstd * g[j];
        m = fmaxf(m, amax8(a));
      }
    }
    m = row_max<kWarps>(m, s_part[1] + group * kWarps, group, warp, lane);
    row_scale = blk::scale_of(m);
    if (tid == 0) static_cast<float*>(p.scales)[row] = row_scale;
  }

#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v = tid + i * kLanes;
    if (i * kLanes >= p.vecs) break;                       // (uniform: the shuffles need every lane)
    const bool mine = v < p.vecs;
    float a[8];
    unpack8(q[i], a);
    if (mine) {
      float g[8];
      load_gain(p.gain, p.gain_fp32, p.gain_offset, v, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = a[j] * rstd * g[j];
      if (p.out != nullptr) p.out[at + v] = pack8(a);
    }
    if (p.form == MOE_FORM_BLK) {                          // 16 lanes hold a block of 128
      float m = amax8(a);
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, off));
      const float sc = blk::scale_of(m);
      uint32_t w[2];
      blk::pack(a, sc, w);
      if (mine) {
        p.codes[at + v] = make_uint2(w[0], w[1]);
        if ((lane & 15) == 0) static_cast<float*>(p.scales)[static_cast<size_t>(v >> 4) * p.rows + row] = sc;
      }
    } else if (p.form == MOE_FORM_MX) {                    // four lanes a block of 32, sixteen a word of scale bytes
      float m = amax8(a);
      m = fmaxf(m, __shfl_xor_sync(kFull, m, 1));
      m = fmaxf(m, __shfl_xor_sync(kFull, m, 2));
      const uint32_t byte = mx::scale_byte(m);
      uint32_t word = byte << (2 * (lane & 12));
      word |= __shfl_xor_sync(kFull, word, 4);
      word |= __shfl_xor_sync(kFull, word, 8);
      const float inv = mx::inverse_scale(byte);
      if (mine) {
        p.codes[at + v] = make_uint2(mx::pack4(a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv),
                                     mx::pack4(a[4] * inv, a[5] * inv, a[6] * inv, a[7] * inv));
        if ((lane & 15) == 0) static_cast<uint32_t*>(p.scales)[static_cast<size_t>(v >> 4) * p.rows + row] = word;
      }
    } else if (p.form == MOE_FORM_ROWS) {
      uint32_t w[2];
      blk::pack(a, row_scale, w);
      if (mine) p.codes[at + v] = make_uint2(w[0], w[1]);
    }
  }
}

// Rows group, group + groups, ...; the columns of a lane are the same in all of them.
template <int kWarps, int kVecs>
__global__ void __launch_bounds__(kWarps * 32 > kBlock ? kWarps * 32 : kBlock)
norm_backward(const NormGradParams p) {
  constexpr int kGroups = kWarps * 32 >= kBlock ? 1 : kBlock / (kWarps * 32);
  constexpr int kLanes = kWarps * 32;
  __shared__ float s_part[4][kGroups * kWarps];
  extern __shared__ float s_gain[];                        // [kGroups - 1][cols]
  const int lane = threadIdx.x & 31, group = threadIdx.x / kLanes, tid = threadIdx.x % kLanes, warp = tid >> 5;
  float acc[kVecs][8];
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;

  int turn = 0;
  for (long long row = static_cast<long long>(blockIdx.x) * kGroups + group; row < p.rows;
       row += static_cast<long long>(gridDim.x) * kGroups) {
    const size_t at = static_cast<size_t>(row) * p.vecs;
    uint4 sq[kVecs], dq[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kLanes;
      sq[i] = dq[i] = make_uint4(0u, 0u, 0u, 0u);
      if (v < p.vecs) {
        sq[i] = p.s[at + v];
        dq[i] = p.d_out[at + v];
      }
    }
    float ss = 0.f, dot = 0.f;                             // sums of s^2 and of s d_out gain
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kLanes;
      if (v < p.vecs) {
        float s[8], d[8], g[8];
        unpack8(sq[i], s);
        unpack8(dq[i], d);
        load_gain(p.gain, p.gain_fp32, p.gain_offset, v, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          ss = fmaf(s[j], s[j], ss);
          dot = fmaf(s[j], d[j] * g[j], dot);
        }
      }
    }
    // two pairs of arrays in turn: a row's reads are over when the next row but one writes (the warps meet in between)
    ss = moe::warp_sum(ss);
    dot = moe::warp_sum(dot);
    if constexpr (kWarps > 1) {
      float* part_s = s_part[2 * turn] + group * kWarps;
      float* part_d = s_part[2 * turn + 1] + group * kWarps;
      if (lane == 0) {
        part_s[warp] = ss;
        part_d[warp] = dot;
      }
      row_sync<kWarps>(group);
      ss = moe::warp_sum(lane < kWarps ? part_s[lane] : 0.f);
      dot = moe::warp_sum(lane < kWarps ? part_d[lane] : 0.f);
      turn ^= 1;
    }
    const float rstd = rstd_of(ss, p.cols, p.eps);
    const float mean = __fdiv_rn(dot * rstd, static_cast<float>(p.cols));   // mean of g h
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kLanes;
      if (v < p.vecs) {
        float s[8], d[8], g[8], o[8];
        unpack8(sq[i], s);
        unpack8(dq[i], d);
        load_gain(p.gain, p.gain_fp32, p.gain_offset, v, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float h = s[j] * rstd;
          acc[i][j] = fmaf(d[j], h, acc[i][j]);
          o[j] = rstd * (d[j] * g[j] - h * mean);
        }
        if (p.d_x != nullptr) {
          if (p.d_sum != nullptr) {
            float a[8];
            unpack8(p.d_sum[at + v], a);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] += a[j];
          }
          p.d_x[at + v] = pack8(o);
        }
      }
    }
  }

  if (p.partial == nullptr) return;
  if constexpr (kGroups > 1) {                             // the CTA's rows in the order of their groups
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * kLanes;
        if (v < p.vecs) {
          float4* d = reinterpret_cast<float4*>(s_gain + static_cast<size_t>(group - 1) * p.cols) + 2 * v;
          d[0] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
          d[1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
        }
      }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kLanes;
      if (v < p.vecs) {
        for (int o = 0; o < kGroups - 1; ++o) {
          const float* src = s_gain + static_cast<size_t>(o) * p.cols + 8 * v;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[i][j] += src[j];
        }
      }
    }
  }
  float4* dst = reinterpret_cast<float4*>(p.partial + static_cast<size_t>(blockIdx.x) * p.cols);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v = tid + i * kLanes;
    if (v < p.vecs) {
      dst[2 * v] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
      dst[2 * v + 1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
    }
  }
}

// d_gain of 32 columns: eight warps take every eighth partial row, then the eight sums in order.
__global__ void __launch_bounds__(kBlock)
norm_gain_sum(const float* __restrict__ partial, int parts, int cols, float* __restrict__ d_gain) {
  __shared__ float s_sum[kBlock / 32][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < cols)
    for (int i = warp; i < parts; i += kBlock / 32) sum += partial[static_cast<size_t>(i) * cols + c];
  s_sum[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && c < cols) {
    sum = 0.f;
    for (int i = 0; i < kBlock / 32; ++i) sum += s_sum[i][lane];
    d_gain[c] = sum;
  }
}

// Warps per row: the smallest power of two with which `vecs` vectors fit, kVecs to a lane.
int warps_of(int vecs, int per_lane) {
  int w = 1;
  while (w < 32 && w * 32 * per_lane < vecs) w *= 2;
  return w;
}
// Vectors per lane: 4, so that a row's loads are in flight together and few warps have to meet.
int vecs_per_lane(int) { return 4; }

// CTAs of norm_backward, the same for its scratch and its launch.
int backward_ctas(const moe_ctx* ctx, long long rows, int vecs) {
  const int lanes = 32 * warps_of(vecs, vecs_per_lane(vecs));
  const int groups = lanes >= kBlock ? 1 : kBlock / lanes;
  const long long need = (rows + groups - 1) / groups, room = static_cast<long long>(ctx->num_sms) * (lanes > kBlock ? 1 : 2);
  return static_cast<int>(need < room ? need : room);
}

template <int kVecs>
cudaError_t launch_norm(const NormParams& p, int warps, cudaStream_t stream) {
  const int groups = warps * 32 >= kBlock ? 1 : kBlock / (warps * 32);
  const int threads = warps * 32 > kBlock ? warps * 32 : kBlock;
  const unsigned grid = static_cast<unsigned>((p.rows + groups - 1) / groups);
  switch (warps) {
    case 1: add_rms_norm<1, kVecs><<<grid, threads, 0, stream>>>(p); break;
    case 2: add_rms_norm<2, kVecs><<<grid, threads, 0, stream>>>(p); break;
    case 4: add_rms_norm<4, kVecs><<<grid, threads, 0, stream>>>(p); break;
    case 8: add_rms_norm<8, kVecs><<<grid, threads, 0, stream>>>(p); break;
    case 16: add_rms_norm<16, kVecs><<<grid, threads, 0, stream>>>(p); break;
    default: add_rms_norm<32, kVecs><<<grid, threads, 0, stream>>>(p); break;
  }
  return cudaGetLastError();
}

template <int kVecs>
cudaError_t launch_backward(const NormGradParams& p, int warps, int ctas, cudaStream_t stream) {
  const int groups = warps * 32 >= kBlock ? 1 : kBlock / (warps * 32);
  const int threads = warps * 32 > kBlock ? warps * 32 : kBlock;
  const size_t smem = p.partial ? static_cast<size_t>(groups - 1) * p.cols * 4 : 0;   // at most 7 x 1024 values
  switch (warps) {
    case 1: norm_backward<1, kVecs><<<ctas, threads, smem, stream>>>(p); break;
    case 2: norm_backward<2, kVecs><<<ctas, threads, smem, stream>>>(p); break;
    case 4: norm_backward<4, kVecs><<<ctas, threads, smem, stream>>>(p); break;
    case 8: norm_backward<8, kVecs><<<ctas, threads, smem, stream>>>(p); break;
    case 16: norm_backward<16, kVecs><<<ctas, threads, smem, stream>>>(p); break;
    default: norm_backward<32, kVecs><<<ctas, threads, smem, stream>>>(p); break;
  }
  return cudaGetLastError();
}

}  // namespace

namespace moe {

cudaError_t launch_add_rms_norm(moe_ctx* ctx, const moe_rms_norm_args& a, cudaStream_t stream) {
  const NormParams p{static_cast<const uint4*>(a.x), static_cast<const uint4*>(a.residual), a.gain,
                     static_cast<uint4*>(a.sum_out), static_cast<uint4*>(a.out), static_cast<uint2*>(a.codes), a.scales,
                     a.rows, a.cols / 8, a.cols, a.eps, a.gain_offset, a.gain_fp32, a.form};
  ctx->last_launches += 1;
  return launch_norm<4>(p, warps_of(p.vecs, 4), stream);
}

size_t rms_norm_scratch_bytes(const moe_ctx* ctx, long long rows, int cols) {
  return static_cast<size_t>(backward_ctas(ctx, rows, cols / 8)) * cols * 4;
}

cudaError_t launch_rms_norm_backward(moe_ctx* ctx, const moe_rms_norm_grad_args& a, cudaStream_t stream) {
  if (a.rows == 0) return a.d_gain ? cudaMemsetAsync(a.d_gain, 0, static_cast<size_t>(a.cols) * 4, stream) : cudaSuccess;
  const int vecs = a.cols / 8, ctas = backward_ctas(ctx, a.rows, vecs);
  const NormGradParams p{static_cast<const uint4*>(a.s), a.gain, static_cast<const uint4*>(a.d_out),
                         static_cast<const uint4*>(a.d_sum), static_cast<uint4*>(a.d_x),
                         a.d_gain ? static_cast<float*>(a.scratch) : nullptr, a.rows, vecs, a.cols, a.eps, a.gain_offset,
                         a.gain_fp32};
  cudaError_t e = launch_backward<4>(p, warps_of(vecs, 4), ctas, stream);
  ctx->last_launches += 1;
  if (e == cudaSuccess && a.d_gain) {
    norm_gain_sum<<<(a.cols + 31) / 32, kBlock, 0, stream>>>(p.partial, ctas, a.cols, a.d_gain);
    ctx->last_launches += 1;
    e = cudaGetLastError();
  }
  return e;
}

}  // namespace moe
