// Residual addition and RMS norm with an output in bf16, in 8 bits with scales, or both; and the norm's gradients.
//
// The statistics are sums over s = bf16(x + residual) as stored: the gradient then sees the same function, from the same tensor.
//
// add_rms_norm  : one row by as few warps as hold it, the row in registers from its one read to its last write.  Without residual
//                 and codes the CTAs stay and load a row ahead.
// norm_backward : the CTAs stay and take every gridDim-th group of rows; the rows to come are on their way into a ring in shared
//                 memory by bulk copies; a lane's columns are the same in all rows, so its gains stay in registers, and the
//                 gain's gradient is summed there: one partial row per CTA, added by norm_gain_sum in a fixed order.
//
// n = s rstd (gain + offset) with rstd = (mean s^2 + eps)^-1/2; with h = s rstd and g = (gain + offset) d_out,
// dx = d_sum + rstd (g - h mean(g h)) and d_gain = sum over rows of d_out h.  All of it fp32; s, out and dx are rounded to bf16
// once, codes from the fp32 n.
//
// Bound by HBM for many rows: 8192 x 7168 with residual, bf16 and 8-bit outputs 85.9 us, 6.2 TB/s (80.8 at the rate of a copy); the
// gradients of 8192 x 4096 54 us, 44 of them norm_backward at 6.1 TB/s, 4.8 norm_gain_sum, the rest between the two.  64 x 7168:
// 4.2 us, of which the launch is half; the gradients of 301 x 7168 12.4 us: two launches of two loads' latency each.  Gradients of
// rows above 8192 columns are bound by registers: up to 32 warps to a row leave a thread 64 for four vectors of three tensors and
// their sums, which spill (4096 x 8192 53 us, 4096 x 9216 286, 4096 x 12288 323; the bytes take 41, 46 and 61).
#include <cuda_bf16.h>

#include "blk_quant.cuh"
#include "moe_internal.h"
#include "mx_quant.cuh"
#include "ptx_sm100.cuh"
#include "route_scored.cuh"

namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kMaxRing = 4;
constexpr int kRingBytes = 216 * 1024;    // of shared memory for the rings of an SM
constexpr int kStayThreads = 3 * 256;     // of an SM, where the forward's CTAs stay

struct NormParams {
  const uint4* x;
  const uint4* residual;
  const void* gain;
  uint4* sum;
  uint4* out;
  uint2* codes;
  void* scales;
  long long rows;
  int vecs, cols;                         // vectors of eight values, and values, of a row
  float eps, gain_offset;
};

struct NormGradParams {
  const uint4* s;
  const void* gain;
  const uint4* d_out;
  const uint4* d_sum;
  uint4* d_x;
  float* partial;                         // [CTAs][cols], or null
  int32_t* status;
  long long rows;
  int vecs, cols;
  float eps, gain_offset;
  int ring;
};

__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// Keeps a vector packed over a point of the program: the compiler would otherwise hold the eight values it once unpacked.
__device__ __forceinline__ void stay_packed(uint4& q) { asm volatile("" : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w)); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}
// x + residual in bf16 pairs: one rounding to nearest even.
__device__ __forceinline__ uint32_t add2(uint32_t x, uint32_t r) {
  const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&r));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 add8(const uint4& x, const uint4& r) {
  return make_uint4(add2(x.x, r.x), add2(x.y, r.y), add2(x.z, r.z), add2(x.w, r.w));
}
__device__ __forceinline__ float squares8(const uint4& q, float ss) {
  float a[8];
  unpack8(q, a);
#pragma unroll
  for (int j = 0; j < 8; ++j) ss = fmaf(a[j], a[j], ss);
  return ss;
}
template <bool kFp32>
__device__ __forceinline__ void load_gain(const void* gain, float offset, int v, float (&g)[8]) {
  if constexpr (kFp32) {
    const float4 a = __ldg(static_cast<const float4*>(gain) + 2 * v), b = __ldg(static_cast<const float4*>(gain) + 2 * v + 1);
    g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w;
    g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
  } else {
    unpack8(__ldg(static_cast<const uint4*>(gain) + v), g);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] += offset;
}

// How a CTA's threads share rows: `warps` warps to a row, `rows` rows to a CTA.
struct Share {
  int warps, rows;
};
// The warps of one row meet (named barriers: a CTA's last rows may be missing).
__device__ __forceinline__ void row_sync(int group, int warps) {
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * warps) : "memory");
}
// Sum over the row's warps in a fixed order.  `part` holds the warps' sums, and zeros up to the eighth.
__device__ __forceinline__ float sum_of(const float* part, int warps, int lane) {
  if (warps <= 8) {
    const float4 a = *reinterpret_cast<const float4*>(part), b = *reinterpret_cast<const float4*>(part + 4);
    return ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
  }
  return moe::warp_sum(lane < warps ? part[lane] : 0.f);
}
// Floats of a row's sums in shared memory.
constexpr int kParts = 32;
// ... for the most rows of a CTA (eight of one warp each take eight floats).
__device__ __forceinline__ float* part_of(float* parts, int group, int warps) { return parts + group * (warps <= 8 ? 8 : kParts); }
constexpr int kPartFloats = 64;

__device__ __forceinline__ float row_max(float v, float* part, int group, int warps, int warp, int lane) {
  v = moe::warp_max(v);
  if (warps > 1) {
    if (lane == 0) part[warp] = v;
    row_sync(group, warps);
    v = moe::warp_max(lane < warps ? part[lane] : 0.f);
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

// kStay: without a residual; the CTAs stay and take every gridDim-th group of rows, the next of which is on its way while one is
// worked on.
template <int kVecs, int kThreads, int kForm, bool kFp32, bool kStay>
__global__ void __launch_bounds__(kThreads, kStay ? kStayThreads / kThreads : kThreads <= 256 ? 4 : 1)
add_rms_norm(const NormParams p, const Share share) {
  __shared__ __align__(16) float s_part[3][kPartFloats];   // sums, in two arrays in turn where the CTA stays, and maxima
  const int lanes = 32 * share.warps, group = threadIdx.x / lanes, tid = threadIdx.x - group * lanes;
  const int lane = tid & 31, warp = tid >> 5;
  long long row = static_cast<long long>(blockIdx.x) * share.rows + group;
  for (int i = threadIdx.x; i < 2 * kPartFloats; i += blockDim.x) s_part[0][i] = 0.f;
  __syncthreads();
  if (row >= p.rows) return;                               // (all warps of a row alike)
  const long long step = static_cast<long long>(gridDim.x) * share.rows;
  auto fetch = [&](uint4 (&to)[kVecs], long long from) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * lanes;
      to[i] = make_uint4(0u, 0u, 0u, 0u);
      if (v < p.vecs) to[i] = p.x[static_cast<size_t>(from) * p.vecs + v];
    }
  };
  uint4 q[kVecs], next[kVecs];
  if constexpr (kStay) fetch(next, row);
  for (int turn = 0;; turn ^= 1) {
    const size_t at = static_cast<size_t>(row) * p.vecs;
    if constexpr (kStay) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) q[i] = next[i];
      if (row + step < p.rows) fetch(next, row + step);
    } else {
      fetch(q, row);
    }
    if (!kStay && p.residual != nullptr) {
      uint4 r[kVecs];
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * lanes;
        r[i] = make_uint4(0u, 0u, 0u, 0u);
        if (v < p.vecs) r[i] = p.residual[at + v];
      }
#pragma unroll
      for (int i = 0; i < kVecs; ++i) q[i] = add8(q[i], r[i]);
    }
    if (p.sum != nullptr) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * lanes;
        if (v < p.vecs) p.sum[at + v] = q[i];
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) ss = squares8(q[i], ss);
    ss = moe::warp_sum(ss);
    if (share.warps > 1) {
      float* part = part_of(s_part[turn], group, share.warps);
      if (lane == 0) part[warp] = ss;
      row_sync(group, share.warps);
      ss = sum_of(part, share.warps, lane);
    }
    const float rstd = rstd_of(ss, p.cols, p.eps);

    float row_scale = 1.f;
    if constexpr (kForm == MOE_FORM_ROWS) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        float a[8], g[8];
        unpack8(q[i], a);
        load_gain<kFp32>(p.gain, p.gain_offset, min(tid + i * lanes, p.vecs - 1), g);
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = a[j] * rstd * g[j];
        m = fmaxf(m, amax8(a));
      }
      m = row_max(m, part_of(s_part[2], group, share.warps), group, share.warps, warp, lane);
      row_scale = blk::scale_of(m);
      if (tid == 0) static_cast<float*>(p.scales)[row] = row_scale;
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * lanes;
      if (i * lanes >= p.vecs) break;                       // (uniform: the shuffles need every lane)
      const bool mine = v < p.vecs;
      // (a lane behind the row works on zeros: what it finds does not count in a maximum, even where it is NaN)
      float a[8], g[8];
      unpack8(q[i], a);
      load_gain<kFp32>(p.gain, p.gain_offset, min(v, p.vecs - 1), g);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = a[j] * rstd * g[j];
      if (p.out != nullptr && mine) p.out[at + v] = pack8(a);
      if constexpr (kForm == MOE_FORM_BLK) {                          // 16 lanes hold a block of 128
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
      } else if constexpr (kForm == MOE_FORM_MX) {                    // four lanes a block of 32, sixteen a word of scale bytes
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
      } else if constexpr (kForm == MOE_FORM_ROWS) {
        uint32_t w[2];
        blk::pack(a, row_scale, w);
        if (mine) p.codes[at + v] = make_uint2(w[0], w[1]);
      }
    }
    if constexpr (!kStay) return;
    row += step;
    if (row >= p.rows) return;
  }
}

// The ring: groups of neighbouring rows of up to three tensors, `depth` groups deep, filled by one thread.
struct Ring {
  uint64_t full[kMaxRing];
  int abort_flag;
};
__device__ __forceinline__ void ring_init(Ring* ring, int depth) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < depth; ++i) ptx::mbar_init(ptx::smem_u32(&ring->full[i]), 1);
    ring->abort_flag = 0;
    ptx::fence_barrier_init();
  }
  __syncthreads();
}
// A wait gave up (never in a sound run): reported, and copies in flight get time to land before the CTA ends.
__device__ __forceinline__ void ring_gave_up(int32_t* status, int where) {
  if (threadIdx.x == 0) {
    atomicCAS(&status[0], 0, MOE_ERR_TIMEOUT);
    atomicCAS(&status[1], 0, where);
  }
  for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}

template <int kThreads, bool kFp32>
__global__ void __launch_bounds__(kThreads, kThreads <= 256 ? 2 : 1)
norm_backward(const NormGradParams p, const Share share) {
  constexpr int kVecs = 4;
  extern __shared__ __align__(16) unsigned char s_ring[];
  __shared__ __align__(16) float s_part[4][kPartFloats];
  __shared__ Ring ring;
  const int lanes = 32 * share.warps, group = threadIdx.x / lanes, tid = threadIdx.x - group * lanes;
  const int lane = tid & 31, warp = tid >> 5, groups = share.rows;
  for (int i = threadIdx.x; i < 4 * kPartFloats; i += blockDim.x) s_part[0][i] = 0.f;
  const bool with_sum = p.d_sum != nullptr && p.d_x != nullptr;
  const uint32_t row_bytes = p.cols * 2, tensor_bytes = groups * row_bytes;
  const uint32_t slot_bytes = with_sum ? 3 * tensor_bytes : 2 * tensor_bytes;
  const long long step = static_cast<long long>(gridDim.x) * groups;
  ring_init(&ring, p.ring);
  auto fill = [&](int slot, long long row) {
    if (row >= p.rows) return;
    const uint32_t bytes = static_cast<uint32_t>(p.rows - row < groups ? p.rows - row : groups) * row_bytes;
    const uint32_t full = ptx::smem_u32(&ring.full[slot]), dst = ptx::smem_u32(s_ring) + slot * slot_bytes;
    ptx::mbar_expect_tx(full, with_sum ? 3 * bytes : 2 * bytes);
    ptx::bulk_load(dst, p.s + row * p.vecs, bytes, full);
    ptx::bulk_load(dst + tensor_bytes, p.d_out + row * p.vecs, bytes, full);
    if (with_sum) ptx::bulk_load(dst + 2 * tensor_bytes, p.d_sum + row * p.vecs, bytes, full);
  };
  long long row0 = static_cast<long long>(blockIdx.x) * groups;
  if (threadIdx.x == 0)
    for (int i = 0; i < p.ring; ++i) fill(i, row0 + i * step);

  // a lane's columns are the same in all rows: its gains stay in registers, where a thread has enough of them (8192 x 4096 53.8 us,
  // 57.5 with the gains read from L1 for each row)
  constexpr bool kKeepGain = kThreads <= 256;
  float acc[kVecs][8], gains[kKeepGain ? kVecs : 1][8];
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
  if constexpr (kKeepGain) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) load_gain<kFp32>(p.gain, p.gain_offset, min(tid + i * lanes, p.vecs - 1), gains[i]);
  }
  auto gain_of = [&](int i, float (&g)[8]) {               // (a lane behind the row multiplies zeros, or is not looked at)
    if constexpr (kKeepGain) {
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = gains[i][j];
    } else {
      load_gain<kFp32>(p.gain, p.gain_offset, min(tid + i * lanes, p.vecs - 1), g);
    }
  };
  int slot = 0, turn = 0;
  uint32_t phase = 0;
  for (; row0 < p.rows; row0 += step) {
    const bool ok = ptx::mbar_wait(ptx::smem_u32(&ring.full[slot]), phase, &ring.abort_flag);
    const long long row = row0 + group;
    const bool live = row < p.rows;
    const size_t at = static_cast<size_t>(row) * p.vecs;
    const uint4* in = reinterpret_cast<const uint4*>(s_ring + slot * slot_bytes + group * row_bytes);
    const int pitch = tensor_bytes / 16;                   // vectors between the tensors' rows
    uint4 sq[kVecs], dq[kVecs], eq[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * lanes;
      sq[i] = dq[i] = eq[i] = make_uint4(0u, 0u, 0u, 0u);
      if (live && v < p.vecs) {
        sq[i] = in[v];
        dq[i] = in[v + pitch];
      }
    }
    if (with_sum) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * lanes;
        if (live && v < p.vecs) eq[i] = in[v + 2 * pitch];
      }
    }
    float ss = 0.f, dot = 0.f;                             // sums of s^2 and of s d_out gain
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float s[8], d[8], g[8];
      unpack8(sq[i], s);
      unpack8(dq[i], d);
      gain_of(i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ss = fmaf(s[j], s[j], ss);
        dot = fmaf(s[j], d[j] * g[j], dot);
      }
    }
    ss = moe::warp_sum(ss);
    dot = moe::warp_sum(dot);
    // two pairs of arrays in turn: a row's reads are over when the next row but one writes (the CTA meets in between)
    float* part_s = part_of(s_part[2 * turn], group, share.warps);
    float* part_d = part_of(s_part[2 * turn + 1], group, share.warps);
    if (share.warps > 1 && lane == 0) {
      part_s[warp] = ss;
      part_d[warp] = dot;
    }
    if (__syncthreads_or(!ok)) {                           // the slot has been read, the warps' sums are written
      ring_gave_up(p.status, 301);
      return;
    }
    if (threadIdx.x == 0) fill(slot, row0 + p.ring * step);
    if (++slot == p.ring) { slot = 0; phase ^= 1u; }
    if (share.warps > 1) {
      ss = sum_of(part_s, share.warps, lane);
      dot = sum_of(part_d, share.warps, lane);
    }
    turn ^= 1;
    const float rstd = rstd_of(ss, p.cols, p.eps);
    const float mean = __fdiv_rn(dot * rstd, static_cast<float>(p.cols));   // mean of g h
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float s[8], d[8], o[8], g[8];
      stay_packed(sq[i]);
      stay_packed(dq[i]);
      unpack8(sq[i], s);
      unpack8(dq[i], d);
      unpack8(eq[i], o);
      gain_of(i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float h = s[j] * rstd;
        acc[i][j] = fmaf(d[j], h, acc[i][j]);
        o[j] = fmaf(rstd, fmaf(-h, mean, d[j] * g[j]), o[j]);
      }
      const int v = tid + i * lanes;
      if (p.d_x != nullptr && live && v < p.vecs) p.d_x[at + v] = pack8(o);
    }
  }

  if (p.partial == nullptr) return;
  if (groups > 1) {                             // the CTA's rows in the order of their groups
    float* s_gain = reinterpret_cast<float*>(s_ring);      // [groups - 1][cols]: the ring is idle
    __syncthreads();
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * lanes;
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
      const int v = tid + i * lanes;
      if (v < p.vecs) {
        for (int o = 0; o < groups - 1; ++o) {
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
    const int v = tid + i * lanes;
    if (v < p.vecs) {
      dst[2 * v] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
      dst[2 * v + 1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
    }
  }
}

// d_gain of 32 columns: the CTA's warps take every kSumWarps-th partial row, then the warps' sums in order.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(kSumWarps * 32)
norm_gain_sum(const float* __restrict__ partial, int parts, int cols, float* __restrict__ d_gain) {
  constexpr int kAhead = 8;                                // rows whose loads are in flight together
  __shared__ float s_sum[kSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < cols) {
    for (int i = warp; i < parts; i += kSumWarps * kAhead) {
      float v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        v[u] = i + u * kSumWarps < parts ? __ldcg(partial + static_cast<size_t>(i + u * kSumWarps) * cols + c) : 0.f;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) sum += v[u];
    }
  }
  s_sum[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && c < cols) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kSumWarps; ++i) sum += s_sum[i][lane];
    d_gain[c] = sum;
  }
}

// As few warps to a row as hold its vectors, `per_lane` to a lane, and as many rows to a CTA as fit into 256 threads.
Share share_of(int vecs, int per_lane) {
  Share s;
  s.warps = (vecs - 1) / (32 * per_lane) + 1;
  s.rows = s.warps >= 8 ? 1 : 8 / s.warps;
  return s;
}
int threads_of(const Share& s) { return 32 * s.warps * s.rows; }

using NormKernel = void (*)(NormParams, Share);
template <int kVecs, int kThreads>
NormKernel norm_kernel(const moe_rms_norm_args& a) {
  switch (a.form) {
    case MOE_FORM_ROWS:
      return a.gain_fp32 ? add_rms_norm<kVecs, kThreads, MOE_FORM_ROWS, true, false>
                         : add_rms_norm<kVecs, kThreads, MOE_FORM_ROWS, false, false>;
    case MOE_FORM_MX:
      return a.gain_fp32 ? add_rms_norm<kVecs, kThreads, MOE_FORM_MX, true, false>
                         : add_rms_norm<kVecs, kThreads, MOE_FORM_MX, false, false>;
    case MOE_FORM_BLK:
      return a.gain_fp32 ? add_rms_norm<kVecs, kThreads, MOE_FORM_BLK, true, false>
                         : add_rms_norm<kVecs, kThreads, MOE_FORM_BLK, false, false>;
    default:
      return a.gain_fp32 ? add_rms_norm<kVecs, kThreads, MOE_FORM_NONE, true, false>
                         : add_rms_norm<kVecs, kThreads, MOE_FORM_NONE, false, false>;
  }
}
NormKernel staying_kernel(const moe_rms_norm_args& a) {
  return a.gain_fp32 ? add_rms_norm<4, 256, MOE_FORM_NONE, true, true> : add_rms_norm<4, 256, MOE_FORM_NONE, false, true>;
}

// norm_backward: the CTAs of an SM that its registers and rings allow, and the rings' depth.  Two CTAs for up to 8192 columns, three
// where a row takes five warps (and a CTA one row): 8192 x 7168 81.8 us against 96.4 with one, 8192 x 4096 53.8 against 53.4; 7774 x
// 4152 49.3 with three against 59.5 with two.
struct BackwardPlan {
  Share share;
  int ctas, depth;
  size_t bytes;                           // of a ring
};
BackwardPlan backward_plan(int cols) {
  BackwardPlan b;
  b.share = share_of(cols / 8, 4);
  const size_t slot = static_cast<size_t>(3) * b.share.rows * cols * 2;   // (as if d_sum were given)
  b.ctas = threads_of(b.share) > 256 || 4 * slot > kRingBytes ? 1 : threads_of(b.share) <= 160 ? 3 : 2;
  b.depth = static_cast<int>(kRingBytes / b.ctas / slot);
  if (b.depth > kMaxRing) b.depth = kMaxRing;
  b.bytes = b.depth * slot;               // (the longest row takes 192 KiB)
  return b;
}
using BackwardKernel = void (*)(NormGradParams, Share);
template <bool kFp32>
BackwardKernel backward_kernel(const BackwardPlan& b) {
  return threads_of(b.share) <= 256 ? norm_backward<256, kFp32> : norm_backward<1024, kFp32>;
}
// CTAs of norm_backward: no more than it takes to be done in as few rounds as all that fit would be, since each leaves a row of
// fp32 sums.  `most`: all that fit, which the scratch is measured by, so that one for many rows does for fewer.
int backward_ctas(const moe_ctx* ctx, long long rows, const BackwardPlan& b, bool most) {
  const long long groups = (rows + b.share.rows - 1) / b.share.rows, room = static_cast<long long>(ctx->num_sms) * b.ctas;
  const long long rounds = most || groups == 0 ? 1 : (groups + room - 1) / room;
  const long long ctas = (groups + rounds - 1) / rounds;
  return static_cast<int>(ctas < room ? ctas : room);
}

}  // namespace

namespace moe {

cudaError_t launch_add_rms_norm(moe_ctx* ctx, const moe_rms_norm_args& a, cudaStream_t stream) {
  const NormParams p{static_cast<const uint4*>(a.x), static_cast<const uint4*>(a.residual), a.gain, static_cast<uint4*>(a.sum_out),
                     static_cast<uint4*>(a.out), static_cast<uint2*>(a.codes), a.scales, a.rows, a.cols / 8, a.cols, a.eps,
                     a.gain_offset};
  ctx->last_launches += 1;
  // Four vectors to a lane keep a row's loads in flight together and few warps meeting; one, where all vectors of the batch are
  // resident at once even so, is quicker done.  64 x 7168: 4.2 us against 6.2; 1000 x 2048: 6.3 / 8.3; 592 x 7168: 10.3 / 8.3.
  const bool few = a.rows * p.vecs <= 2048LL * ctx->num_sms && p.vecs <= 1024;
  const Share share = share_of(p.vecs, few ? 1 : 4);
  const int threads = threads_of(share);
  // Without residual and codes a row has few loads in flight and little to compute: then the CTAs stay and load a row ahead (8192 x
  // 7168 41.3 us against 49.2, 13324 x 2560 26.7 against 34.9).  With codes the registers of the next row cost more (blocks of
  // 128, 8192 x 7168: 84.9 against 69.8).
  const long long groups = (a.rows + share.rows - 1) / share.rows, room = static_cast<long long>(ctx->num_sms) * (kStayThreads / threads);
  const bool stay = a.form == MOE_FORM_NONE && a.residual == nullptr && !few && threads <= 256 && groups > room;
  const long long rounds = stay ? (groups + room - 1) / room : 1;
  auto kernel = stay ? staying_kernel(a) : few ? norm_kernel<1, 1024>(a) : threads <= 256 ? norm_kernel<4, 256>(a) : norm_kernel<4, 1024>(a);
  kernel<<<static_cast<unsigned>((groups + rounds - 1) / rounds), threads, 0, stream>>>(p, share);
  return cudaGetLastError();
}

size_t rms_norm_scratch_bytes(const moe_ctx* ctx, long long rows, int cols) {
  return static_cast<size_t>(backward_ctas(ctx, rows, backward_plan(cols), true)) * cols * 4;
}

cudaError_t launch_rms_norm_backward(moe_ctx* ctx, const moe_rms_norm_grad_args& a, cudaStream_t stream) {
  if (a.rows == 0) return a.d_gain ? cudaMemsetAsync(a.d_gain, 0, static_cast<size_t>(a.cols) * 4, stream) : cudaSuccess;
  const BackwardPlan b = backward_plan(a.cols);
  const int ctas = backward_ctas(ctx, a.rows, b, false), threads = threads_of(b.share);
  const NormGradParams p{static_cast<const uint4*>(a.s), a.gain, static_cast<const uint4*>(a.d_out),
                         static_cast<const uint4*>(a.d_sum), static_cast<uint4*>(a.d_x),
                         a.d_gain ? static_cast<float*>(a.scratch) : nullptr, ctx->d_status, a.rows, a.cols / 8, a.cols, a.eps,
                         a.gain_offset, b.depth};
  // (the ring's bytes also hold the groups' sums of the gain: 4 (rows - 1) cols of at least 6 rows cols)
  auto kernel = a.gain_fp32 ? backward_kernel<true>(b) : backward_kernel<false>(b);
  kernel<<<ctas, threads, b.bytes, stream>>>(p, b.share);
  cudaError_t e = cudaGetLastError();
  ctx->last_launches += 1;
  if (e == cudaSuccess && a.d_gain) {
    norm_gain_sum<<<(a.cols + 31) / 32, kSumWarps * 32, 0, stream>>>(p.partial, ctas, a.cols, a.d_gain);
    ctx->last_launches += 1;
    e = cudaGetLastError();
  }
  return e;
}

cudaError_t prepare_rms_norm(moe_ctx* ctx) {
  (void)ctx;
  cudaError_t e = cudaSuccess;
  for (const int cols : {8192, 32768}) {                   // a plan of each kind
    const BackwardPlan b = backward_plan(cols);
    for (const BackwardKernel kernel : {backward_kernel<false>(b), backward_kernel<true>(b)})
      if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes);
  }
  return e;
}

}  // namespace moe
