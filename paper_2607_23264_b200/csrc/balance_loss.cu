// Balance loss of a router with its per-expert counts, and its gradient.
//
// balance_partial : a CTA per slot of up to kSlotTokens tokens of one sequence, a warp per token; a lane keeps the
//                   probability sums of its experts (lane, lane + 32, ...) in registers over its warp's tokens, the warps are
//                   added in order, the counts are integer atomics in shared memory.  Sequence q has the slots from
//                   offsets[q] / kSlotTokens + q on: no prefix sum over sequences is needed, and the slots of neighbours do
//                   not meet.
// balance_finish  : a CTA per sequence and 32 experts adds the slots' sums, forms the mean and the sequence's share of the
//                   loss; the last CTA to finish adds the shares in order.
// balance_backward: a warp per token: the loss reaches the logits through the counts alone, so one pass over the logits.
#include <climits>

#include "moe_internal.h"
#include "route_scored.cuh"
#include "warp_search.cuh"

namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSlotTokens = 32;
constexpr int kFinishThreads = 1024;

// What a call keeps in its scratch, in 4-byte words: [slots][E] sums, [slots][E] counts, [slots] tokens, [slots] sums of squared
// logarithms, then per sequence and group of 32 experts a share of the loss, per sequence its sum of squares, and the ticket.
struct Scratch {
  float* sums;
  int32_t* counts;
  int32_t* tokens;
  float* z;
  float* share;
  float* seq_z;
  int32_t* ticket;
};
inline long long slots_of(int T, int sequences) { return static_cast<long long>(T) / kSlotTokens + sequences + 1; }
inline size_t scratch_words(int T, int E, int sequences) {
  const size_t slots = static_cast<size_t>(slots_of(T, sequences));
  return slots * (2 * static_cast<size_t>(E) + 2) + static_cast<size_t>(sequences) * ((E + 31) / 32 + 1) + 4;
}
inline Scratch carve(void* base, int T, int E, int sequences) {
  const size_t slots = static_cast<size_t>(slots_of(T, sequences));
  Scratch s;
  s.sums = static_cast<float*>(base);
  s.counts = reinterpret_cast<int32_t*>(s.sums + slots * E);
  s.tokens = s.counts + slots * E;
  s.z = reinterpret_cast<float*>(s.tokens + slots);
  s.share = s.z + slots;
  s.seq_z = s.share + static_cast<size_t>(sequences) * ((E + 31) / 32);
  s.ticket = reinterpret_cast<int32_t*>(s.seq_z + sequences);
  return s;
}

struct BalanceParams {
  const float* logits;
  const int32_t* ids;
  const int32_t* offsets;
  const uint8_t* mask;
  Scratch scratch;
  int32_t* status;
  int T, E, k, sequences, sigmoid;
  float coef, z_coef;
};

__device__ __forceinline__ int offset_at(const int32_t* offsets, int q, int T) {
  if (offsets == nullptr) return q == 0 ? 0 : T;
  const int o = __ldg(offsets + q);
  return min(max(o, 0), T);
}
// Probabilities of one token over its lanes: x becomes p; returns what else the losses need.
struct Token {
  float lse;                                               // log of the sum of exponentials, -inf when all are masked
  bool any;                                                // an expert is left
};
template <int EL>
__device__ __forceinline__ Token probabilities(float (&x)[EL], float (&soft)[EL], bool sigmoid, bool want_soft) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < EL; ++i) top = fmaxf(top, x[i]);
  bool nan = false;
#pragma unroll
  for (int i = 0; i < EL; ++i) nan |= x[i] != x[i];
  top = moe::warp_max(top);
  nan = __any_sync(kFull, nan);
  Token t;
  t.any = top > -INFINITY || nan;
  const float base = top > -INFINITY ? top : 0.f;
  t.lse = -INFINITY;
  if (!sigmoid || want_soft) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      soft[i] = expf(x[i] - base);
      sum += soft[i];
    }
    sum = moe::warp_sum(sum);
    const float inv = t.any ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) soft[i] *= inv;
    if (t.any) t.lse = logf(sum) + base;
  }
  if (sigmoid) {
    // From -40 down sigma(x) is exp(x) to 2^-57, and the shares of the sum are those of exp(x - top), which stays in range.
    const bool far = top < -40.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      x[i] = far ? expf(x[i] - base) : moe::route_sigmoid(x[i]);
      sum += x[i];
    }
    sum = moe::warp_sum(sum);
#pragma unroll
    for (int i = 0; i < EL; ++i) x[i] = t.any ? __fdiv_rn(x[i], sum) : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) x[i] = soft[i];
  }
  return t;
}

template <int EL>
__global__ void __launch_bounds__(kThreads)
balance_partial(const BalanceParams p) {
  extern __shared__ float s_sum[];                         // [kWarps][E] sums, then [E] counts
  __shared__ int s_tokens[kWarps];
  __shared__ float s_z[kWarps];
  int* s_count = reinterpret_cast<int*>(s_sum + kWarps * p.E);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slot = blockIdx.x;
  if (slot == 0 && threadIdx.x == 0) *p.scratch.ticket = 0;
  for (int e = threadIdx.x; e < p.E; e += kThreads) s_count[e] = 0;

  const int q = moe::last_at_or_below(p.sequences, slot, lane, [&](int i) {
    return static_cast<long long>(offset_at(p.offsets, i, p.T) / kSlotTokens) + i;
  });
  int t0 = 0, t1 = 0;
  if (q >= 0) {
    const int begin = offset_at(p.offsets, q, p.T), end = offset_at(p.offsets, q + 1, p.T);
    const long long first = begin + (static_cast<long long>(slot) - (begin / kSlotTokens + q)) * kSlotTokens;
    t0 = static_cast<int>(first < end ? first : end);
    t1 = min(t0 + kSlotTokens, end);
  }
  __syncthreads();

  float acc[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) acc[i] = 0.f;
  float z = 0.f;
  int tokens = 0;
  const bool want_z = p.z_coef != 0.f;
  for (int t = t0 + warp; t < t1; t += kWarps) {
    if (p.mask != nullptr && p.mask[t] == 0) continue;
    const float* row = p.logits + static_cast<size_t>(t) * p.E;
    float x[EL], soft[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const int e = lane + 32 * i;
      x[i] = e < p.E ? __ldg(row + e) : -INFINITY;
    }
    if (lane < p.k) {
      const size_t s = static_cast<size_t>(t) * p.k + lane;
      const int id = p.ids[s];
      if (id >= 0 && id < p.E) {
        atomicAdd(s_count + id, 1);
      } else {
        atomicCAS(&p.status[0], 0, MOE_ERR_BAD_ROUTING);
        atomicCAS(&p.status[1], 0, static_cast<int>(s));
      }
    }
    const Token token = probabilities<EL>(x, soft, p.sigmoid, want_z);
#pragma unroll
    for (int i = 0; i < EL; ++i) acc[i] += x[i];
    if (want_z && token.any) z = fmaf(token.lse, token.lse, z);
    ++tokens;
  }
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    if (e < p.E) s_sum[warp * p.E + e] = acc[i];
  }
  if (lane == 0) {
    s_tokens[warp] = tokens;
    s_z[warp] = z;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += kThreads) {
    float sum = 0.f;
    for (int w = 0; w < kWarps; ++w) sum += s_sum[w * p.E + e];
    p.scratch.sums[static_cast<size_t>(slot) * p.E + e] = sum;
    p.scratch.counts[static_cast<size_t>(slot) * p.E + e] = s_count[e];
  }
  if (threadIdx.x == 0) {
    int n = 0;
    float sum = 0.f;
    for (int w = 0; w < kWarps; ++w) {
      n += s_tokens[w];
      sum += s_z[w];
    }
    p.scratch.tokens[slot] = n;
    p.scratch.z[slot] = sum;
  }
}

__global__ void __launch_bounds__(kFinishThreads)
balance_finish(const BalanceParams p, int slots, int32_t* __restrict__ counts, int32_t* __restrict__ tokens,
               float* __restrict__ mean, float* __restrict__ loss) {
  constexpr int kRows = kFinishThreads / 32;
  __shared__ float s_sum[kRows][33];
  __shared__ int s_count[kRows][33];
  __shared__ int s_tokens[kRows];
  __shared__ float s_z[kRows];
  __shared__ double s_loss[kRows][2];
  __shared__ int s_n[kRows];
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int parts = (p.E + 31) / 32, q = blockIdx.x / parts, part = blockIdx.x % parts, e = part * 32 + lane;
  const int begin = offset_at(p.offsets, q, p.T), end = offset_at(p.offsets, q + 1, p.T);
  const int first = begin / kSlotTokens + q;
  const int used = min(end > begin ? (end - begin + kSlotTokens - 1) / kSlotTokens : 0, slots - first);
  float sum = 0.f, z = 0.f;
  int count = 0, n = 0;
  for (int i = warp; i < used; i += kRows) {
    const size_t at = static_cast<size_t>(first + i);
    if (e < p.E) {
      sum += p.scratch.sums[at * p.E + e];
      count += p.scratch.counts[at * p.E + e];
    }
    n += p.scratch.tokens[at];
    z += p.scratch.z[at];
  }
  s_sum[warp][lane] = sum;
  s_count[warp][lane] = count;
  if (lane == 0) {
    s_tokens[warp] = n;
    s_z[warp] = z;
  }
  __syncthreads();
  if (warp == 0) {
    n = s_tokens[lane];
    z = s_z[lane];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      n += __shfl_xor_sync(kFull, n, off);
      z += __shfl_xor_sync(kFull, z, off);
    }
    sum = 0.f;
    count = 0;
    for (int w = 0; w < kRows; ++w) {
      sum += s_sum[w][lane];
      count += s_count[w][lane];
    }
    float share = 0.f;
    if (e < p.E) {
      const float m = n > 0 ? sum / static_cast<float>(n) : 0.f;
      mean[static_cast<size_t>(q) * p.E + e] = m;
      counts[static_cast<size_t>(q) * p.E + e] = count;
      // a NaN probability shows in the loss whatever the expert's count
      if (n > 0) share = static_cast<float>(count) * p.E / (static_cast<float>(p.k) * static_cast<float>(n)) * m;
    }
    share = moe::warp_sum(share);
    if (lane == 0) {
      p.scratch.share[static_cast<size_t>(q) * parts + part] = share;
      if (part == 0) {
        tokens[q] = n;
        p.scratch.seq_z[q] = z;
      }
      __threadfence();
      s_last = atomicAdd(p.scratch.ticket, 1) == static_cast<int>(gridDim.x) - 1;
    }
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  double total = 0.0, zs = 0.0;
  int all = 0;
  for (long long i = threadIdx.x; i < static_cast<long long>(p.sequences) * parts; i += kFinishThreads)
    total += __ldcg(p.scratch.share + i);
  for (int i = threadIdx.x; i < p.sequences; i += kFinishThreads) {
    zs += __ldcg(p.scratch.seq_z + i);
    all += __ldcg(tokens + i);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    total += __shfl_xor_sync(kFull, total, off);
    zs += __shfl_xor_sync(kFull, zs, off);
    all += __shfl_xor_sync(kFull, all, off);
  }
  if (lane == 0) {
    s_loss[warp][0] = total;
    s_loss[warp][1] = zs;
    s_n[warp] = all;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    total = zs = 0.0;
    all = 0;
    for (int w = 0; w < kRows; ++w) {
      total += s_loss[w][0];
      zs += s_loss[w][1];
      all += s_n[w];
    }
    loss[0] = static_cast<float>(total * p.coef / p.sequences);
    loss[1] = all > 0 ? static_cast<float>(zs * p.z_coef / all) : 0.f;
    tokens[p.sequences] = all;
  }
}

template <int EL>
__global__ void __launch_bounds__(kThreads)
balance_backward(const BalanceParams p, const int32_t* __restrict__ counts, const int32_t* __restrict__ tokens,
                 const float* __restrict__ d_loss, const float* add, float* d_logits) {
  const int lane = threadIdx.x & 31, t = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (t >= p.T) return;
  const size_t at = static_cast<size_t>(t) * p.E;
  float x[EL], soft[EL], d[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    x[i] = e < p.E ? __ldg(p.logits + at + e) : -INFINITY;
    d[i] = add != nullptr && e < p.E ? add[at + e] : 0.f;
  }
  int q = 0;
  if (p.offsets != nullptr) {
    q = moe::last_at_or_below(p.sequences, t, lane, [&](int i) { return static_cast<long long>(offset_at(p.offsets, i, p.T)); });
    if (q < 0 || t >= offset_at(p.offsets, q + 1, p.T)) q = -1;
  }
  if (p.mask != nullptr && p.mask[t] == 0) q = -1;
  const int n = q >= 0 ? __ldg(tokens + q) : 0;
  if (n > 0) {
    const float up = d_loss != nullptr ? __ldg(d_loss) : 1.f;
    const bool want_z = p.z_coef != 0.f;
    float u[EL], own[EL];                                  // own: sigma(-x)
    // coef / sequences E c / (k n) / n, rounded a few times but never out of range where the result is not
    const float f = up * (p.coef / p.sequences) / static_cast<float>(n);
    const float load = static_cast<float>(p.E) / (static_cast<float>(p.k) * static_cast<float>(n));
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const int e = lane + 32 * i;
      u[i] = e < p.E ? f * (load * static_cast<float>(__ldg(counts + static_cast<size_t>(q) * p.E + e))) : 0.f;
      own[i] = p.sigmoid ? moe::route_sigmoid(-x[i]) : 1.f;
    }
    const Token token = probabilities<EL>(x, soft, p.sigmoid, want_z);
    if (token.any) {
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < EL; ++i) dot = fmaf(u[i], x[i], dot);
      dot = moe::warp_sum(dot);
      const float zf = want_z ? up * (2.f * p.z_coef / static_cast<float>(__ldg(tokens + p.sequences))) * token.lse : 0.f;
#pragma unroll
      for (int i = 0; i < EL; ++i) {
        float g = x[i] * (u[i] - dot) * own[i];
        if (want_z) g = fmaf(zf, soft[i], g);
        d[i] += g;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    if (e < p.E) d_logits[at + e] = d[i];
  }
}

BalanceParams params_of(const moe_ctx* ctx, const moe_balance_args& a) {
  const moe_shape& s = ctx->shape;
  BalanceParams p{};
  p.logits = a.logits;
  p.ids = a.topk_ids;
  p.offsets = a.seq_offsets;
  p.mask = a.token_mask;
  p.status = ctx->d_status;
  p.T = s.T;
  p.E = s.E;
  p.k = s.k;
  p.sequences = a.sequences;
  p.sigmoid = a.score == MOE_SCORE_SIGMOID;
  p.coef = a.coef;
  p.z_coef = a.z_coef;
  return p;
}

}  // namespace

namespace moe {

size_t balance_scratch_bytes(const moe_ctx* ctx, int sequences) {
  return (scratch_words(ctx->shape.T, ctx->shape.E, sequences) * 4 + 255) / 256 * 256;
}

cudaError_t launch_balance_loss(moe_ctx* ctx, const moe_balance_args& args, int32_t* counts, int32_t* tokens, float* mean,
                                float* loss, void* scratch, cudaStream_t stream) {
  BalanceParams p = params_of(ctx, args);
  p.scratch = carve(scratch, p.T, p.E, p.sequences);
  const int slots = static_cast<int>(slots_of(p.T, p.sequences));
  const size_t smem = static_cast<size_t>(kWarps + 1) * p.E * 4;          // at most 36 KiB
  auto kernel = p.E <= 32 ? balance_partial<1> : p.E <= 64 ? balance_partial<2> : p.E <= 128 ? balance_partial<4>
                : p.E <= 256 ? balance_partial<8> : p.E <= 512 ? balance_partial<16> : balance_partial<32>;
  kernel<<<slots, kThreads, smem, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  balance_finish<<<static_cast<unsigned>(p.sequences) * ((p.E + 31) / 32), kFinishThreads, 0, stream>>>(
      p, slots, counts, tokens, mean, loss);
  ctx->last_launches += 2;
  return cudaGetLastError();
}

cudaError_t launch_balance_loss_backward(moe_ctx* ctx, const moe_balance_args& args, const int32_t* counts,
                                         const int32_t* tokens, const float* d_loss, const float* add, float* d_logits,
                                         cudaStream_t stream) {
  const BalanceParams p = params_of(ctx, args);
  auto kernel = p.E <= 32 ? balance_backward<1> : p.E <= 64 ? balance_backward<2> : p.E <= 128 ? balance_backward<4>
                : p.E <= 256 ? balance_backward<8> : p.E <= 512 ? balance_backward<16> : balance_backward<32>;
  kernel<<<(p.T + kWarps - 1) / kWarps, kThreads, 0, stream>>>(p, counts, tokens, d_loss, add, d_logits);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

}  // namespace moe
