// The routing plan by a scored rule (moe_plan_routing_scored): selection, histogram, prefixes, stable permutation.
//
// Small batches are planned by one launch, a cluster of eight CTAs: every CTA selects the experts of its eighth of the
// tokens (a warp per token at a time), the histograms of all eight are read through distributed shared memory, and every
// CTA scans the totals and places its own slots.  Larger ones take three launches:
//   1. scored_select : a CTA per chunk of at most 256 slots; a warp per token; the chunk's histogram.
//   2. scored_prefix : a warp per expert; exclusive prefix of the chunk histograms over the chunks, and the total.
//   3. scored_place  : a CTA per chunk; scans the totals over the experts (every CTA for itself: 1024 at most) and places
//                      its slots: (slots of earlier chunks) + (of earlier warps in the chunk) + (of earlier lanes).
// Integer work on decisions that are reproducible bit for bit, so the plan is too.
//
// Bound by instructions, not by bytes: 16384 tokens over 256 experts move 19 MB (2.9 us at the copy rate), and the plan
// takes 34.6 us (graph replay): 27 us of selection, about 1000 warp instructions a token at two thirds of the issue rate,
// then two short launches.  4099 tokens over 96 experts: 15.6 us.  64 tokens over 256 experts, one launch: 7.1 us.
#include <type_traits>

#include "moe_internal.h"
#include "ptx_sm100.cuh"
#include "route_scored.cuh"

namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kWarps = kRouteThreads / 32;
constexpr int kCluster = 8;
// One launch up to this many tokens per CTA of the cluster (four per warp) and one slot per thread; beyond, more CTAs
// selecting side by side are worth two more launches.
constexpr int kSmallTokens = 4 * kWarps;

struct ScoredParams {
  const float* logits;
  const float* bias;
  moe::RouteRule rule;
  int T, E, k;
  int tokens_per_chunk;
  int warp_floats;          // shared memory of a warp's selection
  int32_t* topk_ids;
  float* topk_w;
  int32_t* chunk_hist;      // [chunks][E]
  int32_t* chunk_base;      // [chunks][E]
  int32_t* counts;
  int32_t* offsets;
  int32_t* perm;
  int32_t* inv_perm;
};

// Tokens [t_begin, t_end) of this CTA: ids and weights to global memory, ids to s_ids, their histogram to s_hist (zero).
template <int EL, bool kSigmoid, int kLayout>
__device__ __forceinline__ void select_chunk(const ScoredParams& p, int t_begin, int t_end, int32_t* s_ids, int32_t* s_hist,
                                             float* s_sel) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float next[EL];
  if (t_begin + warp < t_end) moe::load_logits<EL, kLayout>(p.logits + static_cast<size_t>(t_begin + warp) * p.E, p.E, lane, next);
  for (int t = t_begin + warp; t < t_end; t += kWarps) {
    const float* row = p.logits + static_cast<size_t>(t) * p.E;
    float x[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) x[i] = next[i];
    if (t + kWarps < t_end) moe::load_logits<EL, kLayout>(row + static_cast<size_t>(kWarps) * p.E, p.E, lane, next);
    int id;
    float w;
    moe::warp_select_scored<EL, kSigmoid, kLayout>(row, x, p.bias, p.rule, p.E, p.k, lane, s_sel + warp * p.warp_floats, id, w);
    if (lane < p.k) {
      const size_t s = static_cast<size_t>(t) * p.k + lane;
      p.topk_ids[s] = id;
      p.topk_w[s] = w;
      s_ids[(t - t_begin) * p.k + lane] = id;
      atomicAdd(&s_hist[id], 1);              // integer counts: order does not matter
    }
  }
}

// offsets[e] for all experts from their totals, in shared memory (E <= 1024, 256 threads x 4).
__device__ __forceinline__ void scan_totals(const int32_t* s_total, int E, int32_t* s_offset, int32_t* s_warp) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int v[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * tid + i;
    v[i] = e < E ? s_total[e] : 0;
    sum += v[i];
  }
  int incl = sum;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(kFull, incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int run = incl - sum;
  for (int i = 0; i < warp; ++i) run += s_warp[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * tid + i;
    if (e < E) s_offset[e] = run;
    run += v[i];
  }
  __syncthreads();
}

// Places the CTA's slots (at most one per thread, slot numbers from s_begin): s_start[e] = the first row of the CTA's slots
// of expert e; s_warp_cnt [kWarps][E] bytes, zero.
__device__ __forceinline__ void place_slots(const int32_t* s_ids, int n_slots, int s_begin, const int32_t* s_start, int E,
                                            unsigned char* s_warp_cnt, int32_t* perm, int32_t* inv_perm) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool active = tid < n_slots;
  const int e = active ? s_ids[tid] : E + lane;             // idle lanes get distinct keys outside [0, E)
  const unsigned same = __match_any_sync(kFull, e);
  const int before_lane = __popc(same & ((1u << lane) - 1u));
  if (active && before_lane == 0) s_warp_cnt[warp * E + e] = static_cast<unsigned char>(__popc(same));
  __syncthreads();
  if (active) {
    int row = s_start[e] + before_lane;
    for (int i = 0; i < warp; ++i) row += s_warp_cnt[i * E + e];
    perm[row] = s_begin + tid;
    inv_perm[s_begin + tid] = row;
  }
}

template <int EL, bool kSigmoid, int kLayout>
__global__ void __launch_bounds__(kRouteThreads)
scored_select(const ScoredParams p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  int32_t* s_hist = reinterpret_cast<int32_t*>(smem_raw);                 // [E]
  int32_t* s_ids = s_hist + p.E;                                          // [256]
  float* s_sel = reinterpret_cast<float*>(s_ids + kRouteThreads);
  const int t_begin = blockIdx.x * p.tokens_per_chunk, t_end = min(p.T, t_begin + p.tokens_per_chunk);
  for (int e = threadIdx.x; e < p.E; e += kRouteThreads) s_hist[e] = 0;
  __syncthreads();
  select_chunk<EL, kSigmoid, kLayout>(p, t_begin, t_end, s_ids, s_hist, s_sel);
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += kRouteThreads) p.chunk_hist[static_cast<size_t>(blockIdx.x) * p.E + e] = s_hist[e];
}

__global__ void __launch_bounds__(kRouteThreads)
scored_prefix(const ScoredParams p, int chunks) {
  const int lane = threadIdx.x & 31, e = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (e >= p.E) return;
  int run = 0;
  constexpr int kAhead = 16;                                // 32-chunk groups whose loads are in flight together
  for (int c0 = 0; c0 < chunks; c0 += 32 * kAhead) {
    int v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int c = c0 + 32 * u + lane;
      v[u] = c < chunks ? p.chunk_hist[static_cast<size_t>(c) * p.E + e] : 0;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      int incl = v[u];
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(kFull, incl, off);
        if (lane >= off) incl += o;
      }
      const int c = c0 + 32 * u + lane;
      if (c < chunks) p.chunk_base[static_cast<size_t>(c) * p.E + e] = run + incl - v[u];
      run += __shfl_sync(kFull, incl, 31);
    }
  }
  if (lane == 0) p.counts[e] = run;
}

__global__ void __launch_bounds__(kRouteThreads)
scored_place(const ScoredParams p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  int32_t* s_start = reinterpret_cast<int32_t*>(smem_raw);                // [E] totals' scan, then this chunk's first rows
  int32_t* s_total = s_start + p.E;                                       // [E]
  int32_t* s_warp = s_total + p.E;                                        // [8]
  int32_t* s_ids = s_warp + kWarps;                                       // [256]
  unsigned char* s_cnt = reinterpret_cast<unsigned char*>(s_ids + kRouteThreads);   // [8][E]
  const int tid = threadIdx.x, chunk = blockIdx.x;
  const int t_begin = chunk * p.tokens_per_chunk, t_end = min(p.T, t_begin + p.tokens_per_chunk);
  const int n_slots = (t_end - t_begin) * p.k;
  if (tid < n_slots) s_ids[tid] = p.topk_ids[static_cast<size_t>(t_begin) * p.k + tid];
  for (int e = tid; e < p.E; e += kRouteThreads) s_total[e] = p.counts[e];
  for (int i = tid; i < kWarps * p.E; i += kRouteThreads) s_cnt[i] = 0;
  __syncthreads();
  scan_totals(s_total, p.E, s_start, s_warp);
  if (chunk == 0) {
    for (int e = tid; e < p.E; e += kRouteThreads) p.offsets[e] = s_start[e];
    if (tid == 0) p.offsets[p.E] = p.T * p.k;
  }
  __syncthreads();
  for (int e = tid; e < p.E; e += kRouteThreads) s_start[e] += p.chunk_base[static_cast<size_t>(chunk) * p.E + e];
  __syncthreads();
  place_slots(s_ids, n_slots, t_begin * p.k, s_start, p.E, s_cnt, p.perm, p.inv_perm);
}

template <int EL, bool kSigmoid, int kLayout>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kRouteThreads)
scored_plan_small(const ScoredParams p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  int32_t* s_hist = reinterpret_cast<int32_t*>(smem_raw);                 // [E] this CTA's slots per expert
  int32_t* s_start = s_hist + p.E;                                        // [E]
  int32_t* s_total = s_start + p.E;                                       // [E]
  int32_t* s_warp = s_total + p.E;                                        // [8]
  int32_t* s_ids = s_warp + kWarps;                                       // [256]
  float* s_sel = reinterpret_cast<float*>(s_ids + kRouteThreads);
  unsigned char* s_cnt = reinterpret_cast<unsigned char*>(s_sel + kWarps * p.warp_floats);   // [8][E]
  const int tid = threadIdx.x, rank = static_cast<int>(ptx::cluster_ctarank());
  const int t_begin = min(p.T, rank * p.tokens_per_chunk), t_end = min(p.T, t_begin + p.tokens_per_chunk);
  for (int e = tid; e < p.E; e += kRouteThreads) s_hist[e] = 0;
  for (int i = tid; i < kWarps * p.E; i += kRouteThreads) s_cnt[i] = 0;
  __syncthreads();
  select_chunk<EL, kSigmoid, kLayout>(p, t_begin, t_end, s_ids, s_hist, s_sel);
  __syncthreads();
  ptx::cluster_sync();                                      // every CTA's histogram stands
  const uint32_t hist_u32 = ptx::smem_u32(s_hist);
  for (int e = tid; e < p.E; e += kRouteThreads) {
    uint32_t h[kCluster];
#pragma unroll
    for (int c = 0; c < kCluster; ++c) h[c] = ptx::ld_cluster_u32(ptx::map_to_cta(hist_u32 + 4 * e, c));
    int total = 0, before = 0;
#pragma unroll
    for (int c = 0; c < kCluster; ++c) {
      total += h[c];
      before += c < rank ? h[c] : 0;
    }
    s_total[e] = total;
    s_start[e] = before;
  }
  __syncthreads();
  if (rank == 0)
    for (int e = tid; e < p.E; e += kRouteThreads) p.counts[e] = s_total[e];
  // s_hist may not change while other CTAs read it: the scan's result goes over the totals
  ptx::cluster_sync();
  scan_totals(s_total, p.E, s_hist, s_warp);
  if (rank == 0) {
    for (int e = tid; e < p.E; e += kRouteThreads) p.offsets[e] = s_hist[e];
    if (tid == 0) p.offsets[p.E] = p.T * p.k;
  }
  for (int e = tid; e < p.E; e += kRouteThreads) s_start[e] += s_hist[e];
  __syncthreads();
  place_slots(s_ids, (t_end - t_begin) * p.k, t_begin * p.k, s_start, p.E, s_cnt, p.perm, p.inv_perm);
}

// Calls f with the selection's template arguments: entries per lane, sigmoid, layout.
template <typename F>
cudaError_t with_rule(int E, const moe_route_rule& r, F f) {
  auto by_el = [&](auto sigmoid, auto layout) {
    if constexpr (decltype(layout)::value != moe::kOwnGroups) {
      if (E <= 32) return f(std::integral_constant<int, 1>{}, sigmoid, layout);
      if (E <= 64) return f(std::integral_constant<int, 2>{}, sigmoid, layout);
    }
    if (E <= 128) return f(std::integral_constant<int, 4>{}, sigmoid, layout);
    if (E <= 256) return f(std::integral_constant<int, 8>{}, sigmoid, layout);
    if (E <= 512) return f(std::integral_constant<int, 16>{}, sigmoid, layout);
    return f(std::integral_constant<int, 32>{}, sigmoid, layout);
  };
  auto by_layout = [&](auto sigmoid) {
    if (r.n_group == 1) return by_el(sigmoid, std::integral_constant<int, moe::kNoGroups>{});
    // a power of two has no other group sizes, so a lane's share of 4 to 32 neighbours never straddles groups
    if ((E & (E - 1)) == 0 && E >= 128) return by_el(sigmoid, std::integral_constant<int, moe::kOwnGroups>{});
    return by_el(sigmoid, std::integral_constant<int, moe::kAnyGroups>{});
  };
  return r.score == MOE_SCORE_SIGMOID ? by_layout(std::true_type{}) : by_layout(std::false_type{});
}

}  // namespace

namespace moe {

cudaError_t launch_plan_routing_scored(moe_ctx* ctx, const float* logits, const float* bias, const moe_route_rule& rule,
                                       int32_t* topk_ids, float* topk_w, int32_t* counts, int32_t* offsets,
                                       int32_t* perm, int32_t* inv_perm, cudaStream_t stream) {
  const moe_shape& s = ctx->shape;
  ScoredParams p{};
  p.logits = logits;
  p.bias = bias;
  p.rule = make_route_rule(rule, s.E);
  p.T = s.T;
  p.E = s.E;
  p.k = s.k;
  p.warp_floats = route_smem_floats(p.rule);
  p.topk_ids = topk_ids;
  p.topk_w = topk_w;
  p.chunk_hist = ctx->d_chunk_hist;
  p.chunk_base = ctx->d_chunk_base;
  p.counts = counts;
  p.offsets = offsets;
  p.perm = perm;
  p.inv_perm = inv_perm;
  const size_t select_bytes = static_cast<size_t>(kWarps) * p.warp_floats * 4;
  const int per_cta = (s.T + kCluster - 1) / kCluster;
  if (per_cta <= kSmallTokens && per_cta * s.k <= kRouteThreads) {
    p.tokens_per_chunk = per_cta;
    const size_t smem = (3 * static_cast<size_t>(s.E) + kWarps + kRouteThreads) * 4 + select_bytes + kWarps * s.E;
    const cudaError_t e = with_rule(s.E, rule, [&](auto el, auto sigmoid, auto layout) {
      auto kernel = scored_plan_small<decltype(el)::value, decltype(sigmoid)::value, decltype(layout)::value>;
      kernel<<<kCluster, kRouteThreads, smem, stream>>>(p);
      return cudaGetLastError();
    });
    ctx->last_launches += 1;
    moe_mark(ctx, 1, stream);
    moe_mark(ctx, 2, stream);
    moe_mark(ctx, 3, stream);
    return e;
  }
  p.tokens_per_chunk = ctx->tokens_per_chunk;
  const size_t smem1 = (static_cast<size_t>(s.E) + kRouteThreads) * 4 + select_bytes;
  const size_t smem3 = (2 * static_cast<size_t>(s.E) + kWarps + kRouteThreads) * 4 + kWarps * s.E;
  const cudaError_t e = with_rule(s.E, rule, [&](auto el, auto sigmoid, auto layout) {
    auto kernel = scored_select<decltype(el)::value, decltype(sigmoid)::value, decltype(layout)::value>;
    kernel<<<ctx->num_chunks, kRouteThreads, smem1, stream>>>(p);
    return cudaGetLastError();
  });
  if (e != cudaSuccess) return e;
  moe_mark(ctx, 1, stream);
  scored_prefix<<<(s.E + kWarps - 1) / kWarps, kRouteThreads, 0, stream>>>(p, ctx->num_chunks);
  moe_mark(ctx, 2, stream);
  scored_place<<<ctx->num_chunks, kRouteThreads, smem3, stream>>>(p);
  moe_mark(ctx, 3, stream);
  ctx->last_launches += 3;
  return cudaGetLastError();
}

// One-time kernel attributes: the selection's shared memory passes 48 KB at the largest E with many groups.
cudaError_t prepare_plan_scored(moe_ctx* ctx) {
  const int E = ctx->shape.E;
  const moe_route_rule rules[4] = {{MOE_SCORE_SOFTMAX, 1, 1, 1, 0, 1.f}, {MOE_SCORE_SIGMOID, 1, 1, 1, 0, 1.f},
                                   {MOE_SCORE_SOFTMAX, 2, 1, 1, 0, 1.f}, {MOE_SCORE_SIGMOID, 2, 1, 1, 0, 1.f}};
  for (const moe_route_rule& r : rules) {
    const cudaError_t e = with_rule(E, r, [&](auto el, auto sigmoid, auto layout) {
      constexpr int kEl = decltype(el)::value, kL = decltype(layout)::value;
      constexpr bool kS = decltype(sigmoid)::value;
      const cudaError_t a = cudaFuncSetAttribute(scored_select<kEl, kS, kL>, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024);
      if (a != cudaSuccess) return a;
      return cudaFuncSetAttribute(scored_plan_small<kEl, kS, kL>, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024);
    });
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace moe
