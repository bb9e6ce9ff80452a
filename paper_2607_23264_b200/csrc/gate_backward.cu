// Gradients of the gate: the combine's (to the expert rows and the weights) and the scored routing's (to the logits).
//
// combine_backward : one warp per slot (t, j), four where that leaves the SMs short of loads in flight.  They read the
//                    token's d_out row and the slot's y row once, write the slot's d_y row and reduce the dot product
//                    (per-lane partial sums in fp32, a fixed butterfly, then the warps in order).  Algorithmic traffic:
//                    2H(T + R) read, 2HR written.  Bound by HBM: with the routing's gradient, 8192 tokens x 2 experts of
//                    4096 take 63 us (336 MB, 5.3 TB/s); 301 tokens x 8 of 7168 take 23 us (74 MB; the launches and the
//                    first loads' latency count).
// routing_backward : a warp per token.  The chosen experts' part is k values, one per lane; the row of d_logits is
//                    written once, and the chosen entries again by the lanes that hold them.
#include <cuda_bf16.h>

#include "moe_internal.h"
#include "route_scored.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;                 // 16-byte vectors of each row a lane has in flight
constexpr unsigned kFull = 0xFFFFFFFFu;

template <int kWarpsPerSlot>
__global__ void __launch_bounds__(kThreads)
combine_backward(const uint4* __restrict__ d_out, const uint4* __restrict__ y_perm, const int32_t* __restrict__ inv_perm,
                 const float* __restrict__ topk_w, uint4* __restrict__ d_y_perm, float* __restrict__ d_topk_w,
                 long long slots, int k, int vec_per_row) {
  __shared__ float s_part[kThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % kWarpsPerSlot;
  const long long slot = static_cast<long long>(blockIdx.x) * (kThreads / 32 / kWarpsPerSlot) + warp / kWarpsPerSlot;
  if (slot >= slots) return;                                // (all warps of a slot alike)
  const size_t row = static_cast<size_t>(inv_perm[slot]);
  const float w = topk_w[slot];
  const uint4* g = d_out + static_cast<size_t>(slot / k) * vec_per_row;
  const uint4* y = y_perm + row * vec_per_row;
  uint4* d = d_y_perm ? d_y_perm + row * vec_per_row : nullptr;
  float dot = 0.f;
  for (int v0 = part * 32 * kAhead + lane; v0 < vec_per_row; v0 += kWarpsPerSlot * 32 * kAhead) {
    uint4 gv[kAhead], yv[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int v = v0 + 32 * u;
      gv[u] = yv[u] = make_uint4(0u, 0u, 0u, 0u);
      if (v < vec_per_row) {
        gv[u] = __ldg(g + v);
        yv[u] = __ldg(y + v);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int v = v0 + 32 * u;
      const __nv_bfloat162* gp = reinterpret_cast<const __nv_bfloat162*>(&gv[u]);
      const __nv_bfloat162* yp = reinterpret_cast<const __nv_bfloat162*>(&yv[u]);
      uint4 o;
      __nv_bfloat162* op = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 a = __bfloat1622float2(gp[i]), b = __bfloat1622float2(yp[i]);
        dot = fmaf(a.x, b.x, dot);
        dot = fmaf(a.y, b.y, dot);
        op[i] = __floats2bfloat162_rn(w * a.x, w * a.y);
      }
      if (d && v < vec_per_row) d[v] = o;
    }
  }
  dot = moe::warp_sum(dot);
  if constexpr (kWarpsPerSlot > 1) {
    if (lane == 0) s_part[warp] = dot;
    // the warps of the slot only: the last CTA's others may be gone
    asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / kWarpsPerSlot), "r"(32 * kWarpsPerSlot) : "memory");
    dot = 0.f;
    for (int i = 0; i < kWarpsPerSlot; ++i) dot += s_part[warp - part + i];
  }
  if (part == 0 && lane == 0) d_topk_w[slot] = dot;
}

// Lane l holds the logits l, l + 32, ... of the token (EL of them, E <= 32 * EL): the row is read once and written once.
template <int EL>
__global__ void __launch_bounds__(kThreads)
routing_backward(const float* __restrict__ logits, const int32_t* __restrict__ topk_ids,
                 const float* __restrict__ d_topk_w, const moe_route_rule rule, float* __restrict__ d_logits, int T, int E,
                 int k, int32_t* __restrict__ status) {
  const int lane = threadIdx.x & 31;
  const int t = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (t >= T) return;
  const float* row = logits + static_cast<size_t>(t) * E;
  float* out = d_logits + static_cast<size_t>(t) * E;
  const bool sigmoid = rule.score == MOE_SCORE_SIGMOID;

  int id = -1;
  float g = 0.f;
  if (lane < k) {
    const size_t s = static_cast<size_t>(t) * k + lane;
    id = topk_ids[s];
    g = d_topk_w[s] * rule.weight_scale;
    if (id < 0 || id >= E) {
      atomicCAS(&status[0], 0, MOE_ERR_BAD_ROUTING);
      atomicCAS(&status[1], 0, static_cast<int>(s));
      id = -1;
      g = 0.f;
    }
  }
  float x[EL];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    x[i] = e < E ? row[e] : -INFINITY;
  }
  const float xs = id >= 0 ? row[id] : -INFINITY;
#pragma unroll
  for (int i = 0; i < EL; ++i) bad |= x[i] != x[i] || (!sigmoid && x[i] == INFINITY);
  bad = __any_sync(kFull, bad);

  const bool dense = !sigmoid && rule.renormalise == 0;   // every expert has a gradient
  float d, dot = 0.f;
  if (sigmoid) {
    const float s = id >= 0 && xs > -INFINITY ? moe::route_sigmoid(xs) : 0.f;
    // 1 - s as the sigmoid of -x (the difference loses its digits from x = 10 on and is 0 from 17), and each score's share
    // of the sum before anything is multiplied by it (1 / S leaves fp32 where all chosen logits are near -88).  0.1 us of
    // 2.1 more at 301 tokens, 0.5 of 7.0 at 16384 (256 experts, logits in L2).
    float share = s, mean = 0.f;
    if (rule.renormalise) {
      const float sum = moe::warp_sum(s);
      share = sum > 0.f ? s / sum : 0.f;
      mean = moe::warp_sum(g * share);
    }
    d = share * (g - mean) * moe::route_sigmoid(-xs);
  } else if (!dense) {
    float m = moe::warp_max(xs);
    if (m == -INFINITY) m = 0.f;
    const float p = expf(xs - m);
    const float sum = moe::warp_sum(p);
    const float q = sum > 0.f ? p / sum : 0.f;
    d = q * (g - moe::warp_sum(g * q));
  } else {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < EL; ++i) top = fmaxf(top, x[i]);
    top = moe::warp_max(top);
    if (top == -INFINITY) top = 0.f;                       // every expert masked: all probabilities 0
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      x[i] = expf(x[i] - top);
      sum += x[i];
    }
    sum = moe::warp_sum(sum);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const float p = expf(xs - top) * inv;
    dot = moe::warp_sum(g * p);
    d = p * (g - dot);
    dot *= -inv;
  }
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    if (e < E) out[e] = bad ? NAN : dense ? x[i] * dot : 0.f;
  }
  __syncwarp();
  if (id >= 0 && !bad) out[id] = d;
}

}  // namespace

namespace moe {

cudaError_t launch_combine_backward(moe_ctx* ctx, const void* d_out, const void* y_perm, const int32_t* inv_perm,
                                    const float* topk_w, void* d_y_perm, float* d_topk_w, cudaStream_t stream) {
  const moe_shape& s = ctx->shape;
  const long long slots = static_cast<long long>(s.T) * s.k;
  // Both gradients, graph replay, one / four warps per slot: 301 tokens x 8 experts of 7168 (2408 slots) 24.2 / 23.1 us.
  // With more slots every SM has enough loads in flight, and four warps only add their meeting.
  const int warps = slots < 24LL * ctx->num_sms ? 4 : 1, per_block = kThreads / 32 / warps;
  auto kernel = warps == 4 ? combine_backward<4> : combine_backward<1>;
  kernel<<<static_cast<unsigned>((slots + per_block - 1) / per_block), kThreads, 0, stream>>>(
      static_cast<const uint4*>(d_out), static_cast<const uint4*>(y_perm), inv_perm, topk_w,
      static_cast<uint4*>(d_y_perm), d_topk_w, slots, s.k, s.H / 8);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

cudaError_t launch_routing_backward(moe_ctx* ctx, const float* logits, const int32_t* topk_ids, const float* d_topk_w,
                                    const moe_route_rule& rule, float* d_logits, cudaStream_t stream) {
  const moe_shape& s = ctx->shape;
  const int per_block = kThreads / 32;
  auto kernel = s.E <= 32 ? routing_backward<1> : s.E <= 64 ? routing_backward<2> : s.E <= 128 ? routing_backward<4>
                : s.E <= 256 ? routing_backward<8> : s.E <= 512 ? routing_backward<16> : routing_backward<32>;
  kernel<<<(s.T + per_block - 1) / per_block, kThreads, 0, stream>>>(logits, topk_ids, d_topk_w, rule, d_logits, s.T, s.E,
                                                                      s.k, ctx->d_status);
  ctx->last_launches += 1;
  return cudaGetLastError();
}

}  // namespace moe
