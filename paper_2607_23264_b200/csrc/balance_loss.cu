// Balance loss of a router with its per-expert counts, and its gradient.
//
// balance_partial : a CTA per slot of up to `slot_tokens` tokens of one sequence, a warp per token; a lane keeps the probability
//                   sums of its experts in registers over its warp's tokens, the warps are added in order, the counts are
//                   integer atomics in shared memory.  Sequence q has the slots from offsets[q] / slot_tokens + q on: no
//                   prefix sum over sequences is needed, and the slots of neighbours do not meet.
// balance_finish  : a CTA per sequence and 32 experts adds the slots' sums, forms the mean and the sequence's share of the
//                   loss; the last CTA to finish adds the shares in order.  Starts while the first kernel ends.
// balance_backward: a warp per token: the loss reaches the logits through the counts alone, so one pass over the logits.
//                   A warp's tokens are neighbours, and what a sequence gives to all of them stays in registers.
// In both passes the next token's logits are on their way while a token is worked on.
//
// The loss needs p and the counts, the gradient dx = p (u - sum u p) (1 - s for sigmoid scores), u from the counts alone; sums,
// probabilities and loss are fp32, counts exact.  16384 tokens of 256 experts, sigmoid: loss 12.0 us for 17.3 MB (partial 7, the
// rest is finish's loads, its ticket and the last CTA's), gradient 8.9 us for 50 MB, mostly out of L2.  Bound by the chain of a token
// (exponential, reciprocal, sum over the warp: about 0.3 us) at the few tokens of a warp, and by launches; 64 tokens take 12.4 us
// for both.
#include <climits>

#include "moe_internal.h"
#include "ptx_sm100.cuh"
#include "route_scored.cuh"
#include "warp_search.cuh"

namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kThreads = 256, kWarps = kThreads / 32;      // of balance_backward
// Warps of balance_partial: sixteen (16384 tokens of 256 experts, loss and gradient: 22.6 us; 26.8 with eight, 22.6 with 32, which
// take 28.1 against 24.8 for 512 sequences of 64 experts), eight where sixteen rows of sums would not fit into 48 KiB.
__host__ __device__ constexpr int partial_warps(int experts_per_lane) { return experts_per_lane <= 16 ? 16 : 8; }

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
// Tokens of a slot, a multiple of eight: one slot per SM where its sixteen warps then have four tokens or more (balance_finish
// reads half as much: 16384 tokens of 256 experts 12.0 us against 13.4 with two), two where there are fewer (4099 tokens of 64
// experts 7.9 us against 8.7 with one, four 10).
inline int slot_tokens_of(const moe_ctx* ctx) {
  const int per = ctx->shape.T / ((ctx->shape.T >= 64 * ctx->num_sms ? 1 : 2) * ctx->num_sms) + 1;
  return (per + 7) / 8 * 8;
}
// At most so many slots, whatever the tokens of one: grows with T and with the sequences.
inline long long most_slots(const moe_ctx* ctx, int sequences) {
  const long long by_tokens = ctx->shape.T / 8, by_sms = 2LL * ctx->num_sms;
  return (by_tokens < by_sms ? by_tokens : by_sms) + sequences + 1;
}
inline size_t scratch_words(const moe_ctx* ctx, int sequences) {
  const size_t slots = static_cast<size_t>(most_slots(ctx, sequences)), E = ctx->shape.E;
  return slots * (2 * E + 2) + static_cast<size_t>(sequences) * ((E + 31) / 32 + 1) + 4;
}
inline Scratch carve(const moe_ctx* ctx, void* base, int sequences) {
  const size_t slots = static_cast<size_t>(most_slots(ctx, sequences)), E = ctx->shape.E;
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
  int T, E, k, sequences, sigmoid, slot_tokens;
  float coef, z_coef;
};

__device__ __forceinline__ int offset_at(const BalanceParams& p, int q) {
  if (p.offsets == nullptr) return q == 0 ? 0 : p.T;
  const int o = __ldg(p.offsets + q);
  return min(max(o, 0), p.T);
}

// The experts of a lane: kVec neighbours, then those 32 * kVec further.
template <int kVec>
__device__ __forceinline__ int expert_of(int lane, int i) {
  return i / kVec * (32 * kVec) + lane * kVec + i % kVec;
}
template <int EL, int kVec>
__device__ __forceinline__ void load_row(const float* row, int E, int lane, float (&x)[EL], float none) {
#pragma unroll
  for (int i = 0; i < EL; i += kVec) {
    const int e = expert_of<kVec>(lane, i);
    if constexpr (kVec == 4) {                             // (E is a multiple of 4)
      const float4 v = e < E ? *reinterpret_cast<const float4*>(row + e) : make_float4(none, none, none, none);
      x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
    } else {
      x[i] = e < E ? row[e] : none;
    }
  }
}
template <int EL, int kVec>
__device__ __forceinline__ void store_row(float* row, int E, int lane, const float (&x)[EL]) {
#pragma unroll
  for (int i = 0; i < EL; i += kVec) {
    const int e = expert_of<kVec>(lane, i);
    if (e < E) {
      if constexpr (kVec == 4) *reinterpret_cast<float4*>(row + e) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
      else row[e] = x[i];
    }
  }
}

struct Token {
  float lse;                                               // log of the sum of exponentials
  bool any;                                                // an expert is left
};
// x becomes the probabilities of a token, own[i] = sigma(-x_i) (1 for softmax scores), soft the softmax when it is wanted.
// Logits within +-80, the usual ones, need neither their maximum over the warp nor a look at masks: the exponentials and their
// sum stay in range, and NaN passes through.  That holds where every lane's experts exist (bits of `here`); numbers of experts
// that leave some out take the general way: 16384 tokens, sigmoid, loss and gradient, 36 us with 384 experts, 22 with 256.
template <int EL>
__device__ __forceinline__ Token probabilities(float (&x)[EL], float (&own)[EL], float (&soft)[EL], uint32_t here, bool sigmoid,
                                               bool want_soft) {
  constexpr float kNear = moe::kNearSigmoid;
  constexpr uint32_t kAll = EL == 32 ? 0xFFFFFFFFu : (1u << EL) - 1;
  float most = -INFINITY, least = INFINITY;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    most = fmaxf(most, x[i]);
    least = fminf(least, x[i]);
  }
  Token t{0.f, true};
  float base = 0.f;
  const bool near = __all_sync(kFull, most <= kNear && least >= -kNear && here == kAll);
  if (!near) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < EL; ++i) nan |= x[i] != x[i];
    most = moe::warp_max(most);
    t.any = most > -INFINITY || __any_sync(kFull, nan);
    base = most > -INFINITY ? most : 0.f;
  }
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
    if (want_soft && t.any) t.lse = logf(sum) + base;
  }
  if (!sigmoid) {
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      x[i] = soft[i];
      own[i] = 1.f;
    }
    return t;
  }
  float sum = 0.f;
  if (near) {
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const float e = expf(-x[i]);
      x[i] = moe::reciprocal_from_one(1.f + e);
      own[i] = e * x[i];                                   // (1 - s loses its digits where s is near 1)
      sum += x[i];
    }
  } else {
    // Below -80 sigma(x) is exp(x) to 2^-115.  When the largest is below -40 all are exp(x) to 2^-57, and the shares of the sum
    // are those of exp(x - most), which stays in range.
    const bool low = most < -40.f;
    const float shift = low ? base : 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const bool by_exp = low || x[i] < -kNear;
      const float e = expf(by_exp ? x[i] - shift : -x[i]), s = moe::reciprocal_from_one(1.f + e);
      x[i] = by_exp ? e : s;
      own[i] = by_exp ? 1.f : e * s;
      sum += x[i];
    }
  }
  sum = moe::warp_sum(sum);
  const float inv = t.any ? 1.f / sum : 0.f;
#pragma unroll
  for (int i = 0; i < EL; ++i) x[i] *= inv;
  return t;
}
// The experts of a lane that exist, a bit each.
template <int EL, int kVec>
__device__ __forceinline__ uint32_t experts_here(int E, int lane) {
  uint32_t here = 0;
#pragma unroll
  for (int i = 0; i < EL; ++i) here |= (expert_of<kVec>(lane, i) < E ? 1u : 0u) << i;
  return here;
}

template <int EL, int kVec, bool kSigmoid>
__global__ void __launch_bounds__(32 * partial_warps(EL))
balance_partial(const BalanceParams p) {
  constexpr int kWarps = partial_warps(EL), kThreads = 32 * kWarps;
  extern __shared__ __align__(16) float s_sum[];           // [kWarps][E] sums, then [E] counts
  __shared__ int s_tokens[kWarps];
  __shared__ float s_z[kWarps];
  int* s_count = reinterpret_cast<int*>(s_sum + kWarps * p.E);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slot = blockIdx.x;
  ptx::launch_dependents();
  if (slot == 0 && threadIdx.x == 0) *p.scratch.ticket = 0;
  for (int e = threadIdx.x; e < p.E; e += kThreads) s_count[e] = 0;

  const int q = moe::last_at_or_below(p.sequences, slot, lane, [&](int i) {
    return static_cast<long long>(offset_at(p, i) / p.slot_tokens) + i;
  });
  int t0 = 0, t1 = 0;
  if (q >= 0) {
    const int begin = offset_at(p, q), end = offset_at(p, q + 1);
    const long long first = begin + (static_cast<long long>(slot) - (begin / p.slot_tokens + q)) * p.slot_tokens;
    if (first >= begin && first < end) {                   // (below begin: offsets that do not ascend)
      t0 = static_cast<int>(first);
      t1 = min(t0 + p.slot_tokens, end);
    }
  }
  __syncthreads();

  float acc[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) acc[i] = 0.f;
  const uint32_t here = experts_here<EL, kVec>(p.E, lane);
  float z = 0.f;
  int tokens = 0;
  const bool want_z = p.z_coef != 0.f;
  auto counts = [&](int t) { return t < t1 && (p.mask == nullptr || p.mask[t] != 0); };
  int t = t0 + warp;
  while (t < t1 && !counts(t)) t += kWarps;
  float next[EL];
  int next_id = -1;
  auto fetch = [&](int at) {
    if (at < t1) {
      load_row<EL, kVec>(p.logits + static_cast<size_t>(at) * p.E, p.E, lane, next, -INFINITY);
      next_id = lane < p.k ? p.ids[static_cast<size_t>(at) * p.k + lane] : 0;
    }
  };
  fetch(t);
  while (t < t1) {
    float x[EL], own[EL], soft[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) x[i] = next[i];
    const int id = next_id, now = t;
    t += kWarps;
    while (t < t1 && !counts(t)) t += kWarps;
    fetch(t);
    if (lane < p.k) {
      if (id >= 0 && id < p.E) {
        atomicAdd(s_count + id, 1);
      } else {
        atomicCAS(&p.status[0], 0, MOE_ERR_BAD_ROUTING);
        atomicCAS(&p.status[1], 0, now * p.k + lane);
      }
    }
    const Token token = probabilities<EL>(x, own, soft, here, kSigmoid, want_z);
#pragma unroll
    for (int i = 0; i < EL; ++i) acc[i] += x[i];
    if (want_z) z = fmaf(token.lse, token.lse, z);
    ++tokens;
  }
  store_row<EL, kVec>(s_sum + warp * p.E, p.E, lane, acc);
  if (lane == 0) {
    s_tokens[warp] = tokens;
    s_z[warp] = z;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += kThreads) {
    float sum = 0.f;
#pragma unroll
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

// kRows warps, each with every kRows-th slot: 32 for many slots to a sequence (16384 tokens of 256 experts, one sequence: 24.7 us for
// loss and gradient, 28.8 with four), four for few (512 sequences of 32 tokens: 25.4 us, 41.7 with 32).
template <int kRows>
__global__ void __launch_bounds__(kRows * 32)
balance_finish(const BalanceParams p, int slots, int32_t* __restrict__ counts, int32_t* __restrict__ tokens,
               float* __restrict__ mean, float* __restrict__ loss) {
  constexpr int kAhead = 8;                                // slots whose loads are in flight together
  __shared__ float s_sum[kRows][33];
  __shared__ int s_count[kRows][33];
  __shared__ int s_tokens[kRows];
  __shared__ float s_z[kRows];
  __shared__ float s_loss[kRows][2];
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int parts = (p.E + 31) / 32, q = blockIdx.x / parts, part = blockIdx.x % parts, e = part * 32 + lane;
  const int begin = offset_at(p, q), end = offset_at(p, q + 1);
  const int first = begin / p.slot_tokens + q;
  const int used = min(end > begin ? (end - begin + p.slot_tokens - 1) / p.slot_tokens : 0, slots - first);
  ptx::wait_for_previous_kernel();
  float sum = 0.f, z = 0.f;
  int count = 0, n = 0;
  for (int i = warp; i < used; i += kRows * kAhead) {
    float s[kAhead], zs[kAhead];
    int c[kAhead], ns[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const size_t at = static_cast<size_t>(first + i + u * kRows);
      const bool in = i + u * kRows < used;
      s[u] = in && e < p.E ? __ldcg(p.scratch.sums + at * p.E + e) : 0.f;
      c[u] = in && e < p.E ? __ldcg(p.scratch.counts + at * p.E + e) : 0;
      ns[u] = in ? __ldcg(p.scratch.tokens + at) : 0;
      zs[u] = in ? __ldcg(p.scratch.z + at) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      sum += s[u];
      count += c[u];
      n += ns[u];
      z += zs[u];
    }
  }
  s_sum[warp][lane] = sum;
  s_count[warp][lane] = count;
  if (lane == 0) {
    s_tokens[warp] = n;
    s_z[warp] = z;
  }
  __syncthreads();
  if (warp == 0) {
    n = lane < kRows ? s_tokens[lane] : 0;
    z = lane < kRows ? s_z[lane] : 0.f;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) n += __shfl_xor_sync(kFull, n, off);
    z = moe::warp_sum(z);
    sum = 0.f;
    count = 0;
#pragma unroll
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
  // the shares in a fixed order, by one warp when they are few
  const int shares = p.sequences * parts, warps = shares <= 256 ? 1 : kRows;
  if (warp >= warps) return;
  float total = 0.f;
  z = 0.f;
  n = 0;
  for (int i = threadIdx.x; i < shares; i += 32 * warps) total += __ldcg(p.scratch.share + i);
  for (int i = threadIdx.x; i < p.sequences; i += 32 * warps) {
    z += __ldcg(p.scratch.seq_z + i);
    n += __ldcg(tokens + i);
  }
  total = moe::warp_sum(total);
  z = moe::warp_sum(z);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) n += __shfl_xor_sync(kFull, n, off);
  if (warps > 1) {
    if (lane == 0) {
      s_loss[warp][0] = total;
      s_loss[warp][1] = z;
      s_tokens[warp] = n;
    }
    __syncthreads();
    if (warp > 0) return;
    total = moe::warp_sum(lane < kRows ? s_loss[lane][0] : 0.f);
    z = moe::warp_sum(lane < kRows ? s_loss[lane][1] : 0.f);
    n = lane < kRows ? s_tokens[lane] : 0;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) n += __shfl_xor_sync(kFull, n, off);
  }
  if (lane == 0) {
    loss[0] = total * (p.coef / static_cast<float>(p.sequences));
    loss[1] = n > 0 ? z * p.z_coef / static_cast<float>(n) : 0.f;
    tokens[p.sequences] = n;
  }
}

// Warp w takes the tokens [w * chunk, (w + 1) * chunk).  Two CTAs on an SM for up to 512 experts, at 128 registers: 16384 tokens
// of 512 experts, loss and gradient, 45.5 us against 49.8 with one of more registers.
template <int EL, int kVec, bool kSigmoid>
__global__ void __launch_bounds__(kThreads, EL <= 8 ? 3 : EL <= 16 ? 2 : 1)
balance_backward(const BalanceParams p, int chunk, const int32_t* __restrict__ counts, const int32_t* __restrict__ tokens,
                 const float* __restrict__ d_loss, const float* add, float* d_logits) {
  const int lane = threadIdx.x & 31;
  const long long begin = (static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * chunk;
  if (begin >= p.T) return;
  const int t0 = static_cast<int>(begin), t1 = static_cast<int>(begin + chunk < p.T ? begin + chunk : p.T);
  const float up = d_loss != nullptr ? __ldg(d_loss) : 1.f;
  const bool want_z = p.z_coef != 0.f;
  float z_scale = 0.f;
  if (want_z) {
    const int all = __ldg(tokens + p.sequences);
    z_scale = all > 0 ? up * (2.f * p.z_coef / static_cast<float>(all)) : 0.f;
  }
  const uint32_t here = experts_here<EL, kVec>(p.E, lane);
  float u[EL];
  int seq_end = t0, n = 0;                                 // of the sequence that u belongs to; none yet
  float next_x[EL], next_d[EL];
  auto fetch = [&](int t) {
    if (t < t1) {
      const size_t at = static_cast<size_t>(t) * p.E;
      load_row<EL, kVec>(p.logits + at, p.E, lane, next_x, -INFINITY);
      if (add != nullptr) load_row<EL, kVec>(add + at, p.E, lane, next_d, 0.f);
    }
  };
  fetch(t0);
  for (int t = t0; t < t1; ++t) {
    float x[EL], d[EL], own[EL], soft[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      x[i] = next_x[i];
      d[i] = add != nullptr ? next_d[i] : 0.f;
    }
    fetch(t + 1);
    if (t >= seq_end) {                                    // the token's sequence, and what its counts give to every token
      int q = 0;
      if (p.offsets != nullptr)
        q = moe::last_at_or_below(p.sequences, t, lane, [&](int i) { return static_cast<long long>(offset_at(p, i)); });
      n = 0;
      seq_end = p.T;
      if (q >= 0 && t < offset_at(p, q + 1)) {
        seq_end = offset_at(p, q + 1);
        n = __ldg(tokens + q);
      } else if (q < 0) {
        seq_end = t + 1;
      }
      if (n > 0) {
        // coef / sequences, E c / (k n) and 1 / n, none of them out of range where the result is not
        const float f = up * (p.coef / p.sequences) / static_cast<float>(n);
        const float load = static_cast<float>(p.E) / (static_cast<float>(p.k) * static_cast<float>(n));
#pragma unroll
        for (int i = 0; i < EL; ++i) {
          const int e = expert_of<kVec>(lane, i);
          u[i] = e < p.E ? f * (load * static_cast<float>(__ldg(counts + static_cast<size_t>(q) * p.E + e))) : 0.f;
        }
      }
    }
    if (n > 0 && (p.mask == nullptr || p.mask[t] != 0)) {
      const Token token = probabilities<EL>(x, own, soft, here, kSigmoid, want_z);
      if (token.any) {
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < EL; ++i) dot = fmaf(u[i], x[i], dot);
        dot = moe::warp_sum(dot);
        const float zf = z_scale * token.lse;
#pragma unroll
        for (int i = 0; i < EL; ++i) {
          float g = x[i] * (u[i] - dot) * own[i];
          if (want_z) g = fmaf(zf, soft[i], g);
          d[i] += g;
        }
      }
    }
    store_row<EL, kVec>(d_logits + static_cast<size_t>(t) * p.E, p.E, lane, d);
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
  p.slot_tokens = slot_tokens_of(ctx);
  p.coef = a.coef;
  p.z_coef = a.z_coef;
  return p;
}

// Four neighbouring experts to a lane where that fills the warp and keeps 16-byte rows: 256 experts 24.7 us for loss and gradient of
// 16384 tokens, 26.4 with single ones; 64 experts, in half a warp, 28.5 against 25.4.
#define MOE_BALANCE_KERNEL(kernel, E, S)                                                                                    \
  ((E) % 4 == 0 && (E) >= 128                                                                                               \
       ? ((E) <= 128 ? kernel<4, 4, S> : (E) <= 256 ? kernel<8, 4, S> : (E) <= 512 ? kernel<16, 4, S> : kernel<32, 4, S>)   \
       : ((E) <= 32 ? kernel<1, 1, S> : (E) <= 64 ? kernel<2, 1, S> : (E) <= 128 ? kernel<4, 1, S>                          \
          : (E) <= 256 ? kernel<8, 1, S> : (E) <= 512 ? kernel<16, 1, S> : kernel<32, 1, S>))

}  // namespace

namespace moe {

size_t balance_scratch_bytes(const moe_ctx* ctx, int sequences) {
  return (scratch_words(ctx, sequences) * 4 + 255) / 256 * 256;
}

cudaError_t launch_balance_loss(moe_ctx* ctx, const moe_balance_args& args, int32_t* counts, int32_t* tokens, float* mean,
                                float* loss, void* scratch, cudaStream_t stream) {
  BalanceParams p = params_of(ctx, args);
  p.scratch = carve(ctx, scratch, p.sequences);
  const int slots = p.T / p.slot_tokens + p.sequences + 1;
  const int warps = partial_warps(p.E <= 512 ? 16 : 32);
  const size_t smem = static_cast<size_t>(warps + 1) * p.E * 4;           // at most 36 KiB
  auto kernel = p.sigmoid ? MOE_BALANCE_KERNEL(balance_partial, p.E, true) : MOE_BALANCE_KERNEL(balance_partial, p.E, false);
  kernel<<<slots, 32 * warps, smem, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  const bool long_ = slots >= 16 * static_cast<long long>(p.sequences);   // many slots to a sequence: more warps share them
  cfg.gridDim = dim3(static_cast<unsigned>(p.sequences) * ((p.E + 31) / 32));
  cfg.blockDim = dim3(long_ ? 1024 : 128);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  ctx->last_launches += 2;
  return cudaLaunchKernelEx(&cfg, long_ ? balance_finish<32> : balance_finish<4>, p, slots, counts, tokens, mean, loss);
}

cudaError_t launch_balance_loss_backward(moe_ctx* ctx, const moe_balance_args& args, const int32_t* counts,
                                         const int32_t* tokens, const float* d_loss, const float* add, float* d_logits,
                                         cudaStream_t stream) {
  const BalanceParams p = params_of(ctx, args);
  // neighbouring tokens of a warp: up to 256 experts all warps are resident at once (16384 tokens of 256 experts, loss and gradient:
  // 24.7 us; 27.2 with half as many warps, 25.9 with twice as many); above, an SM holds 16 or 8 of the 24
  const int chunk = (p.T - 1) / (24 * ctx->num_sms) + 1;
  const int per_block = kWarps * chunk;
  auto kernel = p.sigmoid ? MOE_BALANCE_KERNEL(balance_backward, p.E, true) : MOE_BALANCE_KERNEL(balance_backward, p.E, false);
  kernel<<<(p.T - 1) / per_block + 1, kThreads, 0, stream>>>(p, chunk, counts, tokens, d_loss, add, d_logits);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

}  // namespace moe
