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
__device__ __forceinline__ float route_sigmoid(float x) { return __frcp_rn(1.0f + expf(-x)); }

// 1 / d, correctly rounded, for 1 <= d < 2^116 without the branches of a general reciprocal: nothing leaves the normal range,
// and one step of Newton's method takes the approximate reciprocal to the correctly rounded one
// (tests/exact_arithmetic.cu compares all 2^23 mantissas at several exponents).
__device__ __forceinline__ float reciprocal_from_one(float d) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(d));
  return fmaf(fmaf(-d, y, 1.0f), y, y);
}

// The same bits as route_sigmoid for x >= -kNearSigmoid.
constexpr float kNearSigmoid = 80.0f;
__device__ __forceinline__ float route_sigmoid_near(float x) { return reciprocal_from_one(1.0f + expf(-x)); }

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

// A rule with what the kernels need of it per expert: expert e is in group (e * inv_size) >> 20 (exact for e < 1024: the
// rounded-up reciprocal is off by less than 1 / (2^20 / size) per expert), `lanes` lanes scan a group, and a group starts
// every `pitch` floats in the warp's shared memory (pitch = size + lanes: lanes of different groups read different banks).
struct RouteRule {
  moe_route_rule r;
  int size, lanes, pitch;
  uint32_t inv_size;
};
inline RouteRule make_route_rule(const moe_route_rule& r, int E) {
  RouteRule q{r, E / r.n_group, 32, 0, 0};
  while (q.lanes * r.n_group > 32) q.lanes >>= 1;
  q.pitch = q.size + q.lanes;
  q.inv_size = ((1u << 20) + q.size - 1) / q.size;
  return q;
}
// Floats of shared memory a warp needs for the selection: the groups' ranking values and the list of kept groups.
inline int route_smem_floats(const RouteRule& q) { return q.r.n_group > 1 ? q.r.n_group * q.pitch + 32 : 0; }

// Top k of EL keys per lane (key[i] of the expert expert[i], rising with i and, across lanes, with the candidate index
// lane + 32 i; 0 = none): every lane sorts its own, then k rounds take the largest head.  Lane j returns slot j's expert.
// Ties go to the lower candidate index, hence to the lower expert.
template <int EL>
__device__ __forceinline__ int warp_topk(uint32_t (&key)[EL], int (&expert)[EL], int k, int lane) {
  constexpr unsigned kFull = 0xFFFFFFFFu;
  int id = 0;
  if constexpr (EL <= 8) {
    // odd-even transposition on neighbours with a strict comparison: stable, so equal keys keep the lower expert first
#pragma unroll
    for (int round = 0; round < EL; ++round)
#pragma unroll
      for (int i = round & 1; i + 1 < EL; i += 2) {
        const bool swap = key[i + 1] > key[i];
        const uint32_t ka = swap ? key[i + 1] : key[i], kb = swap ? key[i] : key[i + 1];
        const int ea = swap ? expert[i + 1] : expert[i], eb = swap ? expert[i] : expert[i + 1];
        key[i] = ka; key[i + 1] = kb; expert[i] = ea; expert[i + 1] = eb;
      }
    for (int j = 0; j < k; ++j) {
      const uint32_t largest = __reduce_max_sync(kFull, key[0]);
      const uint32_t heads = __ballot_sync(kFull, key[0] == largest);
      int pick;
      if (__popc(heads) == 1) pick = __shfl_sync(kFull, expert[0], __ffs(heads) - 1);
      else pick = __reduce_min_sync(kFull, key[0] == largest ? expert[0] : 0x7FFFFFFF);
      if (lane == j) id = pick;
      if (key[0] == largest && expert[0] == pick) {        // the owner's next
#pragma unroll
        for (int i = 0; i + 1 < EL; ++i) { key[i] = key[i + 1]; expert[i] = expert[i + 1]; }
        key[EL - 1] = 0u;
      }
    }
  } else {
    for (int j = 0; j < k; ++j) {
      uint32_t best = 0u;
      int best_e = 0x7FFFFFFF;
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (key[i] > best) { best = key[i]; best_e = expert[i]; }
      const uint32_t largest = __reduce_max_sync(kFull, best);
      const int pick = __reduce_min_sync(kFull, best == largest ? best_e : 0x7FFFFFFF);
      if (lane == j) id = pick;
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (expert[i] == pick) key[i] = 0u;
    }
  }
  return id;
}

// The candidates of the kept groups, EL per lane (in ascending expert order), and their top k.
template <int EL>
__device__ __forceinline__ int warp_topk_of_groups(const float* __restrict__ row, const RouteRule& q, bool by_score,
                                                   int count, int k, int lane, const float* rank, const int* kept) {
  uint32_t key[EL];
  int expert[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int c = lane + 32 * i;
    key[i] = 0u;
    expert[i] = 0x7FFFFFFF;
    if (c < count) {
      const int at = static_cast<int>((c * q.inv_size) >> 20), in = c - at * q.size;
      const int g = kept[at];
      expert[i] = g * q.size + in;
      float v = rank[g * q.pitch + in];
      if (by_score) {                                      // ranked by scores, chosen by logits (NaN among the masked)
        v = row[expert[i]];
        if (v != v) v = -INFINITY;
      }
      key[i] = order_key(v);
    }
  }
  return warp_topk<EL>(key, expert, k, lane);
}

// The top k of `count` keys in shared memory, as indexes into them.
template <int EL>
__device__ __forceinline__ int warp_topk_of_keys(const uint32_t* keys, int count, int k, int lane) {
  uint32_t key[EL];
  int at[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    at[i] = lane + 32 * i;
    key[i] = at[i] < count ? keys[at[i]] : 0u;
  }
  return warp_topk<EL>(key, at, k, lane);
}

// How a lane holds a row, and how the groups are found:
//   kNoGroups   lane l holds the logits l, l + 32, ...: one group.
//   kAnyGroups  the same; the groups' members come together in shared memory.
//   kOwnGroups  lane l holds the EL logits from l EL on, which all are of its group (E = 32 EL, a power of two groups): a
//               group is ranked in its lanes' registers, and only the kept groups' keys go through shared memory.
//               16384 tokens over 256 experts in 8 groups, 4 kept: plan 34.6 us, its selection 27 us; with kAnyGroups
//               40.4 and 33 us.  64 tokens: 7.1 and 8.9 us.
enum RouteLayout { kNoGroups, kAnyGroups, kOwnGroups };

// The EL logits of a lane.
template <int EL, int kLayout>
__device__ __forceinline__ void load_logits(const float* __restrict__ row, int E, int lane, float (&x)[EL]) {
  if constexpr (kLayout == kOwnGroups) {
#pragma unroll
    for (int i = 0; i < EL; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(row + lane * EL + i);
      x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const int e = lane + 32 * i;
      x[i] = e < E ? row[e] : -INFINITY;
    }
  }
}

// x: load_logits of the row.  `mem` is route_smem_floats floats of shared memory of this warp.  Lane j < k returns slot
// j's expert and weight.
template <int EL, bool kSigmoid, int kLayout>
__device__ __forceinline__ void warp_select_scored(const float* __restrict__ row, const float (&x)[EL],
                                                   const float* __restrict__ bias, const RouteRule& q, int E, int k,
                                                   int lane, float* mem, int& id, float& w) {
  constexpr unsigned kFull = 0xFFFFFFFFu;
  const moe_route_rule& r = q.r;
  bool bad = false, far = false;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    bad |= x[i] != x[i] || (!kSigmoid && x[i] == INFINITY);
    far |= x[i] < -kNearSigmoid && x[i] > -INFINITY;
  }
  bad = __any_sync(kFull, bad);

  // softmax: largest logit and the sum of the exponentials (fp32; exponents are at most 0), where a score is used
  float top = 0.f, total = 1.f;
  if (!kSigmoid) {
    top = x[0];
#pragma unroll
    for (int i = 1; i < EL; ++i) top = fmaxf(top, x[i]);
    top = warp_max(top);
    if (top == -INFINITY) top = 0.f;               // every expert masked: all exponentials are 0
    if (bias != nullptr || r.renormalise == 0) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < EL; ++i) sum += expf(x[i] - top);
      total = warp_sum(sum);
    }
  }

  // choice values; NaN ranks with the masked experts
  float c[EL];
  if (bias != nullptr) {
    float b[EL];
    load_logits<EL, kLayout>(bias, E, lane, b);
    if (kSigmoid && !__any_sync(kFull, far)) {
#pragma unroll
      for (int i = 0; i < EL; ++i) c[i] = x[i] > -INFINITY ? route_sigmoid_near(x[i]) + b[i] : -INFINITY;
    } else {
#pragma unroll
      for (int i = 0; i < EL; ++i)
        c[i] = x[i] > -INFINITY ? (kSigmoid ? route_sigmoid(x[i]) : __fdiv_rn(expf(x[i] - top), total)) + b[i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < EL; ++i) c[i] = c[i] != c[i] ? -INFINITY : c[i];
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) c[i] = x[i] != x[i] ? -INFINITY : x[i];
  }

  if constexpr (kLayout == kNoGroups) {
    uint32_t key[EL];
    int expert[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      expert[i] = lane + 32 * i;
      key[i] = expert[i] < E ? order_key(c[i]) : 0u;       // 0 is below every key
    }
    id = warp_topk<EL>(key, expert, k, lane);
  } else if constexpr (kLayout == kOwnGroups) {
    const bool by_score = bias == nullptr && r.group_top == 2;   // ranked by scores, chosen by logits
    const int g = lane / q.lanes, sub = lane - g * q.lanes;
    float v1 = -INFINITY, v2 = -INFINITY;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      float v = c[i];
      if (by_score && v > -INFINITY) v = kSigmoid ? route_sigmoid(x[i]) : expf(x[i] - top);
      merge_top2(v1, v2, v, -INFINITY);
    }
    for (int off = q.lanes >> 1; off > 0; off >>= 1) {
      const float b1 = __shfl_xor_sync(kFull, v1, off), b2 = __shfl_xor_sync(kFull, v2, off);
      merge_top2(v1, v2, b1, b2);
    }
    // a group's worth (a masked second expert adds nothing) and its place among the groups, ties to the lower group; the
    // group's lanes share the comparisons
    float worth = v1;
    if (r.group_top == 2 && v2 > -INFINITY) worth = v1 + v2;
    const uint32_t key = order_key(worth);
    int better = 0;
    for (int h0 = 0; h0 < r.n_group; h0 += q.lanes) {
      const int h = h0 + sub;
      const uint32_t other = __shfl_sync(kFull, key, (h * q.lanes) & 31);
      better += h < r.n_group && (other > key || (other == key && h < g)) ? 1 : 0;
    }
    for (int off = q.lanes >> 1; off > 0; off >>= 1) better += __shfl_xor_sync(kFull, better, off);
    const bool stays = better < r.topk_group;
    const uint32_t staying = __ballot_sync(kFull, stays);
    uint32_t* keys = reinterpret_cast<uint32_t*>(mem);
    int* kept = reinterpret_cast<int*>(mem + r.n_group * q.pitch);
    if (stays) {                                                 // the kept groups' keys side by side
      const int at = __popc(staying & ((1u << lane) - 1u));      // lanes of kept groups below this one
      if (sub == 0) kept[at / q.lanes] = g;
#pragma unroll
      for (int i = 0; i < EL; i += 4)
        *reinterpret_cast<uint4*>(keys + at * EL + i) =
            make_uint4(order_key(c[i]), order_key(c[i + 1]), order_key(c[i + 2]), order_key(c[i + 3]));
    }
    __syncwarp();
    const int count = r.topk_group * q.size;
    if (count <= 32) id = warp_topk_of_keys<1>(keys, count, k, lane);
    else if (EL >= 2 && count <= 64) id = warp_topk_of_keys<2>(keys, count, k, lane);
    else if (EL >= 4 && count <= 128) id = warp_topk_of_keys<4>(keys, count, k, lane);
    else id = warp_topk_of_keys<EL>(keys, count, k, lane);
    if (id >= count) id = count - 1;
    const int at = id / q.size;
    id += (kept[at] - at) * q.size;
    __syncwarp();
  } else {
    // what the groups are ranked by, to shared memory in group order
    const bool by_score = bias == nullptr && r.group_top == 2;
    int* kept = reinterpret_cast<int*>(mem + r.n_group * q.pitch);
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const int e = lane + 32 * i;
      if (e < E) {
        float v = c[i];
        if (by_score && v > -INFINITY) v = kSigmoid ? route_sigmoid(x[i]) : expf(x[i] - top);
        mem[e + ((e * q.inv_size) >> 20) * q.lanes] = v;
      }
    }
    __syncwarp();
    // `lanes` lanes per group (a power of two), each scanning every lanes-th expert of it
    const int g = lane / q.lanes, sub = lane - g * q.lanes;
    float v1 = -INFINITY, v2 = -INFINITY;
    if (g < r.n_group) {
      const float* mine = mem + g * q.pitch;
      for (int m = sub; m < q.size; m += q.lanes) merge_top2(v1, v2, mine[m], -INFINITY);
    }
    for (int off = q.lanes >> 1; off > 0; off >>= 1) {
      const float b1 = __shfl_xor_sync(kFull, v1, off), b2 = __shfl_xor_sync(kFull, v2, off);
      merge_top2(v1, v2, b1, b2);
    }
    // a group's worth (a masked second expert adds nothing) and its place among the groups, ties to the lower group
    float worth = v1;
    if (r.group_top == 2 && v2 > -INFINITY) worth = v1 + v2;
    const uint32_t key = order_key(worth);
    int better = 0;
    for (int h = 0; h < r.n_group; ++h) {
      const uint32_t other = __shfl_sync(kFull, key, h * q.lanes);
      better += (other > key || (other == key && h < g)) ? 1 : 0;
    }
    const bool stays = g < r.n_group && sub == 0 && better < r.topk_group;
    const uint32_t staying = __ballot_sync(kFull, stays);
    if (stays) kept[__popc(staying & ((1u << lane) - 1u))] = g;
    __syncwarp();
    const int count = r.topk_group * q.size;
    if (count <= 32) id = warp_topk_of_groups<1>(row, q, by_score, count, k, lane, mem, kept);
    else if (EL >= 2 && count <= 64) id = warp_topk_of_groups<2>(row, q, by_score, count, k, lane, mem, kept);
    else if (EL >= 4 && count <= 128) id = warp_topk_of_groups<4>(row, q, by_score, count, k, lane, mem, kept);
    else id = warp_topk_of_groups<EL>(row, q, by_score, count, k, lane, mem, kept);
    __syncwarp();
  }
  if (id >= E) id = E - 1;                         // nothing left (cannot happen for an allowed k): stay in range

  // weights from the unbiased scores of the chosen
  const float xs = lane < k ? row[id] : -INFINITY;
  float s;
  if (kSigmoid) {
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

}  // namespace moe
