// Scored top-k selection of one token by one warp: softmax or sigmoid scores, a balance bias on the choice, the best
// groups first, weights from the unbiased scores.  The rules are those of moe_plan_routing_scored.
#pragma once
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/moe.h"
#include "route_select.cuh"

namespace moe {

// 1 / (1 + e^-x) with correctly rounded operations around expf: the choice compares these values, so they are the ones
// a plain fp32 program computes, not an approximation of them.
__device__ __forceinline__ float route_sigmoid(float x) { return __fdiv_rn(1.0f, 1.0f + expf(-x)); }

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, off));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
  return v;
}

// The two largest of {a1 >= a2} and {b1 >= b2}.
__device__ __forceinline__ void merge_top2(float& a1, float& a2, float b1, float b2) {
  a2 = fmaxf(fminf(a1, b1), fmaxf(a2, b2));
  a1 = fmaxf(a1, b1);
}

// Lane l holds the logits l, l + 32, ... (EL per lane, E <= 32 * EL).  `rank` is E floats of shared memory of this
// warp, used when there are groups.  Lane j < k returns slot j's expert and weight.
template <int EL>
__device__ __forceinline__ void warp_select_scored(const float* __restrict__ row, const float* __restrict__ bias,
                                                   const moe_route_rule& r, int E, int k, int lane, float* rank, int& id,
                                                   float& w) {
  constexpr unsigned kFull = 0xFFFFFFFFu;
  const bool sigmoid = r.score == MOE_SCORE_SIGMOID;
  float x[EL];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    x[i] = e < E ? row[e] : -INFINITY;
    bad |= x[i] != x[i] || (!sigmoid && x[i] == INFINITY);
  }
  bad = __any_sync(kFull, bad);

  // softmax: largest logit and the sum of the exponentials (fp32; exponents are at most 0)
  float top = 0.f, total = 1.f;
  if (!sigmoid) {
    top = x[0];
#pragma unroll
    for (int i = 1; i < EL; ++i) top = fmaxf(top, x[i]);
    top = warp_max(top);
    if (top == -INFINITY) top = 0.f;               // every expert masked: all exponentials are 0
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) sum += expf(x[i] - top);
    total = warp_sum(sum);
  }

  // choice values, and what the groups are ranked by
  const bool by_score = bias == nullptr && r.n_group > 1 && r.group_top == 2;
  float c[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    c[i] = x[i];
    if (bias != nullptr && e < E && x[i] > -INFINITY)
      c[i] = (sigmoid ? route_sigmoid(x[i]) : __fdiv_rn(expf(x[i] - top), total)) + bias[e];
    if (c[i] != c[i]) c[i] = -INFINITY;            // NaN ranks with the masked experts
    if (r.n_group > 1 && e < E)
      rank[e] = !by_score || x[i] == -INFINITY ? c[i] : sigmoid ? route_sigmoid(x[i]) : expf(x[i] - top);
  }
  uint32_t kept = 0xFFFFFFFFu;                     // bit g: group g stays
  if (r.n_group > 1) {
    __syncwarp();
    // a power of two of lanes per group, each scanning every lanes-th expert of it; the start is rotated by the group
    // so that lanes of different groups read different banks
    const int size = E / r.n_group;
    int lanes = 32;
    while (lanes * r.n_group > 32) lanes >>= 1;
    const int g = lane / lanes, sub = lane % lanes;
    float v1 = -INFINITY, v2 = -INFINITY;
    if (g < r.n_group) {
      const int steps = (size + lanes - 1) / lanes;
      int i = g % steps;
      for (int n = 0; n < steps; ++n) {
        const int m = sub + i * lanes;
        if (m < size) merge_top2(v1, v2, rank[g * size + m], -INFINITY);
        if (++i == steps) i = 0;
      }
    }
    for (int off = lanes >> 1; off > 0; off >>= 1) {
      const float b1 = __shfl_xor_sync(kFull, v1, off), b2 = __shfl_xor_sync(kFull, v2, off);
      merge_top2(v1, v2, b1, b2);
    }
    // worth of the group, held by its first lane; a masked second expert adds nothing
    float worth = v1;
    if (r.group_top == 2 && v2 > -INFINITY) worth = v1 + v2;
    uint32_t key = (g < r.n_group && sub == 0) ? order_key(worth) : 0u;
    kept = 0u;
    for (int j = 0; j < r.topk_group; ++j) {
      const uint32_t best = __reduce_max_sync(kFull, key);
      const int pick = __reduce_min_sync(kFull, key == best ? g : 0x7FFFFFFF);
      kept |= 1u << pick;
      if (g == pick) key = 0u;
    }
    __syncwarp();
  }

  uint32_t key[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    bool open = e < E;
    if (r.n_group > 1 && open) open = (kept >> (e / (E / r.n_group))) & 1u;
    key[i] = open ? order_key(c[i]) : 0u;          // 0 is below every key
  }
  id = 0;
  for (int j = 0; j < k; ++j) {
    uint32_t best = 0;
    int best_e = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < EL; ++i)
      if (key[i] > best) { best = key[i]; best_e = lane + 32 * i; }
    const uint32_t largest = __reduce_max_sync(kFull, best);
    int pick = __reduce_min_sync(kFull, best == largest ? best_e : 0x7FFFFFFF);
    if (pick >= E) pick = E - 1;                   // nothing left (cannot happen for an allowed k): stay in range
#pragma unroll
    for (int i = 0; i < EL; ++i)
      if (pick == lane + 32 * i) key[i] = 0u;
    if (lane == j) id = pick;
  }

  // weights from the unbiased scores of the chosen
  const float xs = lane < k ? row[id] : -INFINITY;
  float s;
  if (sigmoid) {
    s = xs > -INFINITY ? route_sigmoid(xs) : 0.f;
  } else if (r.renormalise) {
    float m = warp_max(xs);                        // relative to the largest chosen logit: never all underflowed
    if (m == -INFINITY) m = 0.f;
    s = expf(xs - m);
  } else {
    s = total > 0.f ? __fdiv_rn(expf(xs - top), total) : 0.f;
  }
  if (r.renormalise) {
    const float sum = warp_sum(s);
    s = sum > 0.f ? __fdiv_rn(s, sum) : 0.f;
  }
  w = bad ? NAN : s * r.weight_scale;
}

__device__ __forceinline__ void warp_select_scored_any(const float* row, const float* bias, const moe_route_rule& r, int E,
                                                       int k, int lane, float* rank, int& id, float& w) {
  if (E <= 32) warp_select_scored<1>(row, bias, r, E, k, lane, rank, id, w);
  else if (E <= 64) warp_select_scored<2>(row, bias, r, E, k, lane, rank, id, w);
  else if (E <= 128) warp_select_scored<4>(row, bias, r, E, k, lane, rank, id, w);
  else if (E <= 256) warp_select_scored<8>(row, bias, r, E, k, lane, rank, id, w);
  else if (E <= 512) warp_select_scored<16>(row, bias, r, E, k, lane, rank, id, w);
  else warp_select_scored<32>(row, bias, r, E, k, lane, rank, id, w);
}

}  // namespace moe
