// Low-rank adapters of many requests added to a projection's output: y[r] += scale_i b_i (a_i x[r]), i the row's adapter.
//
// adapter_rows: short segments and single tokens, where the factors are the bytes.  A cluster of up to eight CTAs takes a unit: up
//               to 16 rows of one adapter out of a window of 256 neighbouring rows, so that a factor is read once for all of
//               them.  The cluster finds its unit by itself: the rows of an adapter are counted, the first, the 17th, ... of
//               them leads a unit, and units are numbered by their leaders.  Each CTA has a part of K and a range of columns.
//               t = x a^T: m16n8k16 products with both operands straight from global memory (a lane's 16 bytes of a row are
//               eight neighbouring k; as x and a are permuted along k alike, no shuffle is needed), warps added in order
//               through shared memory, and the sums sent to every CTA of the cluster.  Then y += t b^T by the same products, t
//               as two bf16 terms: 16 bits of it, since one term's rounding would be as large as the output's.
//
// Bound by latencies: the search for the unit (about 1 us), a's and x's first lines, the exchange of the sums (2 us), b's and y's
// lines.  64 tokens of 32 adapters, rank 16, 7168 -> 4096: 8.4 us, 1.6 TB/s of the 13.5 MB; 1501 rows in 40 uneven segments,
// rank 24, 4112 -> 2104: 18.5 us.
// Long segments take adapter_tiles.
#include <cmath>

#include "adapters.cuh"
#include "ptx_sm100.cuh"

namespace {

using moe::AdapterParams;

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kRows = 16;                 // rows of a unit
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWindow = kThreads;         // rows among which those of one adapter are brought together
constexpr int kMaxCluster = 8;

// The adapter of a row, -1 without one.
__device__ __forceinline__ int adapter_of_row(const AdapterParams& p, long long row, bool report) {
  if (row >= p.rows) return -1;
  int seg = static_cast<int>(row);
  if (p.offsets != nullptr) {
    int lo = -1, hi = p.segments;                          // the last segment that begins at or before the row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(p.offsets + mid) <= row) lo = mid;
      else hi = mid;
    }
    if (lo < 0 || row >= __ldg(p.offsets + lo + 1)) return -1;
    seg = lo;
  }
  const int id = __ldg(p.adapter_of + seg);
  if (id >= p.adapters) {
    if (report) {
      atomicCAS(&p.status[0], 0, MOE_ERR_BAD_ROUTING);
      atomicCAS(&p.status[1], 0, seg);
    }
    return -1;
  }
  return id < 0 ? -1 : id;
}

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// y + d in bf16.
__device__ __forceinline__ uint32_t add_pair(uint32_t y, float d0, float d1) { return moe::pair(moe::low(y) + d0, moe::high(y) + d1); }
// The NaN of eight sums formed again: y + t b, b with the first of the eight columns.  What is NaN by y, t or b is soon given up.
__device__ __forceinline__ uint4 sums_again(const uint4 y, uint4 sum, const float* t, const __nv_bfloat16* b, int rank) {
  float all = 0.f;
#pragma unroll 1
  for (int j = 0; j < rank; ++j) all += fabsf(t[j]);
  if (all != all) return sum;
  const uint32_t old[4] = {y.x, y.y, y.z, y.w};
  uint32_t w[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[2] = {moe::low(w[i]), moe::high(w[i])};
    if (!moe::has_nan(w[i])) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float was = h == 0 ? moe::low(old[i]) : moe::high(old[i]);
      if (v[h] == v[h] || was != was) continue;
      float d = 0.f;
#pragma unroll 1
      for (int j = 0; j < rank && d == d; j += 8) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(b + static_cast<size_t>(2 * i + h) * rank + j));
        const uint32_t qs[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) d = fmaf(t[j + 2 * u + 1], moe::high(qs[u]), fmaf(t[j + 2 * u], moe::low(qs[u]), d));
      }
      v[h] = was + d;
    }
    w[i] = moe::pair(v[0], v[1]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void prefetch_l2(const void* at) { asm volatile("prefetch.global.L2 [%0];" ::"l"(at)); }

// Shared memory: [kWarps][kRows][pitch] sums of the warps, [kRows][pitch] t, [cluster][kRows][pitch] sums of the CTAs.
__host__ __device__ constexpr int pitch_of(int rank) { return rank + 4; }
int smem_of(int rank, int cluster) { return (kWarps + cluster + 1) * kRows * pitch_of(rank) * 4; }

// kTiles: tiles of eight ranks held in registers (rank <= 8 * kTiles).  Grid: for each window `units` clusters.  Above 64 ranks one
// CTA to an SM has the registers (rank 128, 64 tokens of 32 adapters, 4096 x 4096: 24.6 us; 41.1 at half as many, which spill).
template <int kTiles>
__global__ void __launch_bounds__(kThreads, kTiles <= 8 ? 2 : 1)
adapter_rows(const AdapterParams p, int units, int cluster) {
  extern __shared__ float4 smem4[];
  __shared__ __align__(16) int s_id[kWindow];
  __shared__ int s_row[kRows], s_leaders[kWarps], s_unit[2];
  float* s_warp = reinterpret_cast<float*>(smem4);
  const int pitch = pitch_of(p.rank);
  float* s_t = s_warp + kWarps * kRows * pitch;
  float* s_cta = s_t + kRows * pitch;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int item = blockIdx.x / cluster, part = blockIdx.x - item * cluster;
  const int at_window = item / units, unit = item - at_window * units;
  const long long window = static_cast<long long>(at_window) * kWindow;
  const int eighths = p.N / 8;
  const int n0 = 8 * static_cast<int>(static_cast<long long>(eighths) * part / cluster);
  const int n1 = 8 * static_cast<int>(static_cast<long long>(eighths) * (part + 1) / cluster);

  // the window's units: how many rows of its adapter are in front of each row, and the leaders' numbers
  const int my_id = adapter_of_row(p, window + tid, unit == 0 && part == 0);
  s_id[tid] = my_id;
  if (tid < kRows) s_row[tid] = 0;
  if (tid == 0) s_unit[0] = -1;
  const int rows = p.rows - window < kWindow ? static_cast<int>(p.rows - window) : kWindow;
  const bool some_without = __syncthreads_or(tid < rows && my_id < 0);
  int place = __popc(__match_any_sync(kFull, my_id) & ((1u << lane) - 1));
  if (32 * warp < rows) {
    const int4* ids4 = reinterpret_cast<const int4*>(s_id);
#pragma unroll 8
    for (int i = 0; i < 8 * warp; ++i) {
      const int4 v = ids4[i];
      place += (v.x == my_id) + (v.y == my_id) + (v.z == my_id) + (v.w == my_id);
    }
  }
  const bool leads = my_id >= 0 && place % kRows == 0;
  const unsigned leaders = __ballot_sync(kFull, leads);
  if (lane == 0) s_leaders[warp] = __popc(leaders);
  __syncthreads();
  int number = __popc(leaders & ((1u << lane) - 1));
  for (int w = 0; w < warp; ++w) number += s_leaders[w];
  if (leads && number == unit) {
    s_unit[0] = my_id;
    s_unit[1] = place;
  }
  __syncthreads();
  const int id = s_unit[0], first = s_unit[1];
  // rows without an adapter are copied, every units-th by this cluster
  if (some_without && p.y_in != p.y_out) {
    for (int r = unit; r < rows; r += units) {
      if (s_id[r] >= 0) continue;
      const uint4* from = reinterpret_cast<const uint4*>(p.y_in + (window + r) * p.N + n0);
      uint4* to = reinterpret_cast<uint4*>(p.y_out + (window + r) * p.N + n0);
      for (int i = tid; i < (n1 - n0) / 8; i += kThreads) to[i] = from[i];
    }
  }
  if (id < 0) return;                                      // fewer units than clusters (the whole cluster alike)
  const bool mine = my_id == id && place >= first && place < first + kRows;
  if (mine) s_row[place - first] = tid;
  const int count = __syncthreads_count(mine);
  if (cluster > 1) ptx::cluster_arrive();                  // (waited for before anything is sent: every CTA has begun)
  // the bytes of the second product are on their way meanwhile
  {
    const char* b = reinterpret_cast<const char*>(p.b + (static_cast<size_t>(id) * p.N + n0) * p.rank);
    const int bytes = (n1 - n0) * p.rank * 2;
    for (int i = tid * 128; i < bytes; i += kThreads * 128) prefetch_l2(b + i);
  }

  // ------------------------------------------------------------------------------------------------ t = x a^T
  const int steps = (p.K + 31) / 32, tiles = p.rank / 8;   // steps of 32 along K, dealt to the CTAs and then to the warps
  const int s0 = static_cast<int>(static_cast<long long>(steps) * part / cluster);
  const int s1 = static_cast<int>(static_cast<long long>(steps) * (part + 1) / cluster);
  const bool has_lo = g < count, has_hi = g + 8 < count;
  const __nv_bfloat16* x_lo = p.x + (window + (has_lo ? s_row[g] : 0)) * p.K + c * 8;
  const __nv_bfloat16* x_hi = p.x + (window + (has_hi ? s_row[g + 8] : 0)) * p.K + c * 8;
  const __nv_bfloat16* a_row = p.a + (static_cast<size_t>(id) * p.rank + g) * p.K + c * 8;
  float acc[kTiles][4];
#pragma unroll
  for (int j = 0; j < kTiles; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
  // Steps whose loads are in flight together, as far as registers go: rank 16, 64 tokens of 32 adapters 8.5 us against 9.3 with two
  // and 10.2 with one; rank 32, 256 tokens of 32 adapters 14.5 us against 15.2 with four; rank 64 16.5 against 18.2 with two.
  constexpr int kAhead = kTiles <= 2 ? 4 : kTiles <= 4 ? 2 : 1;
  for (int s = s0 + warp; s < s1; s += kWarps * kAhead) {
    uint4 xa[kAhead], xb[kAhead], w[kAhead][kTiles];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = (s + u * kWarps) * 32;
      const bool in = s + u * kWarps < s1 && k + c * 8 < p.K;
      xa[u] = xb[u] = make_uint4(0u, 0u, 0u, 0u);
      if (in && has_lo) xa[u] = __ldg(reinterpret_cast<const uint4*>(x_lo + k));
      if (in && has_hi) xb[u] = __ldg(reinterpret_cast<const uint4*>(x_hi + k));
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        w[u][j] = make_uint4(0u, 0u, 0u, 0u);
        if (in && j < tiles) w[u][j] = __ldg(reinterpret_cast<const uint4*>(a_row + static_cast<size_t>(8 * j) * p.K + k));
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        mma_bf16(acc[j], xa[u].x, xb[u].x, xa[u].y, xb[u].y, w[u][j].x, w[u][j].y);
        mma_bf16(acc[j], xa[u].z, xb[u].z, xa[u].w, xb[u].w, w[u][j].z, w[u][j].w);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    if (j < tiles) {
      float* dst = s_warp + (warp * kRows + g) * pitch + 8 * j + 2 * c;
      *reinterpret_cast<float2*>(dst) = make_float2(acc[j][0], acc[j][1]);
      *reinterpret_cast<float2*>(dst + 8 * pitch) = make_float2(acc[j][2], acc[j][3]);
    }
  }
  __syncthreads();
  if (cluster > 1) ptx::cluster_wait();
  const int quads = p.rank / 4;
  const uint32_t slot = ptx::smem_u32(s_cta) + part * kRows * pitch * 4;
  for (int i = tid; i < count * quads; i += kThreads) {
    const int r = i / quads, j = 4 * (i - r * quads);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < kWarps; ++q) {
      const float4 a = *reinterpret_cast<const float4*>(s_warp + (q * kRows + r) * pitch + j);
      v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
    }
    const uint4 bits = *reinterpret_cast<const uint4*>(&v);
    for (int q = 0; q < cluster; ++q) moe::st_cluster(ptx::map_to_cta(slot + (r * pitch + j) * 4, q), bits);
  }
  // The first of b and y are on their way meanwhile.  A warp takes 32 columns at a time, as four products of eight: in product j
  // a lane's two columns are 2 j and 2 j + 1 of the eight neighbours it keeps, so that it reads and writes 16 bytes of a row.
  constexpr int kSteps = kTiles / 2;                       // steps of 16 ranks
  auto rank_of = [](int s, int lane4) { return kTiles == 2 ? 4 * lane4 : 32 * (s / 2) + 8 * lane4 + 4 * (s % 2); };
  const int groups = (n1 - n0 + 31) / 32;
  const size_t y_lo = static_cast<size_t>(window + (has_lo ? s_row[g] : 0)) * p.N;
  const size_t y_hi = static_cast<size_t>(window + (has_hi ? s_row[g + 8] : 0)) * p.N;
  const __nv_bfloat16* b_base = p.b + static_cast<size_t>(id) * p.N * p.rank;
  uint32_t b[4][2 * kSteps];
  uint4 y[2];
  auto load_group = [&](int at) {
    const int n = n0 + 32 * at;
    y[0] = y[1] = make_uint4(0u, 0u, 0u, 0u);
    if (has_lo && n + 8 * c < n1) y[0] = *reinterpret_cast<const uint4*>(p.y_in + y_lo + n + 8 * c);
    if (has_hi && n + 8 * c < n1) y[1] = *reinterpret_cast<const uint4*>(p.y_in + y_hi + n + 8 * c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = n + (g >> 1) * 8 + 2 * j + (g & 1);
      const __nv_bfloat16* from = b_base + static_cast<size_t>(row) * p.rank;
      if constexpr (kTiles == 2) {
        uint2 v = make_uint2(0u, 0u);
        if (row < n1 && 4 * c < p.rank) v = __ldg(reinterpret_cast<const uint2*>(from + 4 * c));
        b[j][0] = v.x;
        b[j][1] = v.y;
      } else {
#pragma unroll
        for (int s = 0; s < kSteps / 2; ++s) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (row < n1 && 32 * s + 8 * c < p.rank) v = __ldg(reinterpret_cast<const uint4*>(from + 32 * s + 8 * c));
          b[j][4 * s] = v.x;
          b[j][4 * s + 1] = v.y;
          b[j][4 * s + 2] = v.z;
          b[j][4 * s + 3] = v.w;
        }
      }
    }
  };
  if (warp < groups) load_group(warp);
  __syncwarp();
  if (cluster > 1) ptx::cluster_sync();
  else __syncthreads();
  const float f = p.scale != nullptr ? __ldg(p.scale + id) : 1.f;
  for (int i = tid; i < count * quads; i += kThreads) {
    const int r = i / quads, j = 4 * (i - r * quads);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q = 0; q < cluster; ++q) {
      const float4 a = *reinterpret_cast<const float4*>(s_cta + (q * kRows + r) * pitch + j);
      v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
    }
    *reinterpret_cast<float4*>(s_t + r * pitch + j) = make_float4(f * v.x, f * v.y, f * v.z, f * v.w);
  }
  __syncthreads();

  // ------------------------------------------------------------------------------------------------ y += t b^T
  uint32_t hi[kSteps][4], lo[kSteps][4];                   // the terms of t, in the order in which b's lanes hold the ranks
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {                          // rows g and g + 8
#pragma unroll
      for (int e = 0; e < 2; ++e) {                          // ranks 0, 1 and 2, 3 of the step
        const int k = rank_of(s, c) + 2 * e;
        const float* t = s_t + (g + 8 * h) * pitch + k;
        const bool in = g + 8 * h < count && k < p.rank;
        moe::two_terms(in ? t[0] : 0.f, in ? t[1] : 0.f, hi[s][2 * e + h], lo[s][2 * e + h]);
      }
    }
  }
  for (int at = warp; at < groups; at += kWarps) {
    if (at != warp) load_group(at);
    float acc_y[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc_y[j][0] = acc_y[j][1] = acc_y[j][2] = acc_y[j][3] = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        mma_bf16(acc_y[j], hi[s][0], hi[s][1], hi[s][2], hi[s][3], b[j][2 * s], b[j][2 * s + 1]);
        mma_bf16(acc_y[j], lo[s][0], lo[s][1], lo[s][2], lo[s][3], b[j][2 * s], b[j][2 * s + 1]);
      }
    }
    const int n = n0 + 32 * at + 8 * c;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if ((h == 0 ? has_lo : has_hi) && n < n1) {
        const uint4 q = y[h];
        uint4 v = make_uint4(add_pair(q.x, acc_y[0][2 * h], acc_y[0][2 * h + 1]), add_pair(q.y, acc_y[1][2 * h], acc_y[1][2 * h + 1]),
                             add_pair(q.z, acc_y[2][2 * h], acc_y[2][2 * h + 1]), add_pair(q.w, acc_y[3][2 * h], acc_y[3][2 * h + 1]));
        if (moe::has_nan(moe::largest(moe::largest(v.x, v.y, v.z), v.w, v.w)))
          v = sums_again(q, v, s_t + (g + 8 * h) * pitch, b_base + static_cast<size_t>(n) * p.rank, p.rank);
        *reinterpret_cast<uint4*>(p.y_out + (h == 0 ? y_lo : y_hi) + n) = v;
      }
    }
  }
}

// Units of a window at most: an adapter's n rows make (n + 15) / 16 of them.
int units_of(long long rows, int adapters, int segments) {
  const int window = static_cast<int>(rows < kWindow ? rows : kWindow), distinct = adapters < segments ? adapters : segments;
  const int units = distinct + window / kRows;
  return units < 1 ? 1 : units < window ? units : window;
}
// CTAs of a cluster: as many as are resident at once when clusters without a unit are left out.  What is to be expected of a window of n
// rows: s segments that choose among A adapters leave A (1 - e^(-s/A)) of them, and those make (n + 15 distinct) / 16 units at most.
// At 4096 x 4096 (us with 2 / 4 / 8 CTAs to a unit, the choice in brackets): 256 tokens of 32 adapters, rank 32, 12.4 (4) / 14.5 with
// 8; 200 tokens of 100, rank 16, 15.1 (2) / 20.5 with 4; rank 128, 64 tokens of 32 adapters 18.6 (4) / 24.7 with 8.
int cluster_of(long long rows, int segments, bool offsets, int adapters, int rank) {
  const double most = rank > 64 ? 160 : 320;               // (one CTA to an SM, or two; a few more do no harm)
  auto units = [&](double n) {
    const double s = offsets ? n * segments / rows + 1 : n;
    return (n + 15 * adapters * (1 - exp(-s / adapters))) / 16;
  };
  const double all = static_cast<double>(rows / kWindow) * units(kWindow) + (rows % kWindow ? units(static_cast<double>(rows % kWindow)) : 0);
  int c = kMaxCluster;
  while (c > 1 && all * c > most) c /= 2;
  return c;
}
// Whether tiles of 128 rows are quicker.  A unit of 16 rows reads a factor again, so the rows' cost grows with the rank; a tile costs
// the same with few rows in it, and fifteen microseconds to come through.  Above 64 ranks a unit's sums and registers leave an SM
// room for one CTA.  Measured at 4096 x 4096, 8 adapters (rows / tiles, us).  Rank 16: 1024 rows in segments of 256 14 / 20, 4096
// rows in segments of 64 38 / 43, of 128 36 / 36, of 256 36 / 29.  Rank 64: 256 rows 15 / 19, 1024 rows in segments of 64 30 / 23,
// 4096 rows in segments of 16 99 / 104, of 64 62 / 47, of 256 59 / 33.  Rank 128: 256 rows in segments of 8 31 / 30, of 32
// 30 / 20, 4096 rows in segments of 8 168 / 315, of 32 131 / 99, of 256 129 / 44.
bool tiles_are_quicker(const moe_adapter_args& a) {
  if (!a.offsets || a.segments == 0) return false;
  const bool one_cta = a.rank > 64;
  const long long cost = one_cta ? 2 * a.rank : a.rank;
  return a.rows / a.segments * cost >= 4096 && a.rows * cost >= (one_cta ? 40960 : 65536);
}

}  // namespace

namespace moe {

size_t adapter_scratch_bytes(const moe_ctx*, long long, int, int) { return 0; }

moe_status launch_add_adapters(moe_ctx* ctx, const moe_adapter_args& a, cudaStream_t stream) {
  const AdapterParams p{static_cast<const __nv_bfloat16*>(a.x), static_cast<const __nv_bfloat16*>(a.a),
                        static_cast<const __nv_bfloat16*>(a.b), a.scale, a.offsets, a.adapter_of,
                        static_cast<const __nv_bfloat16*>(a.y_in), static_cast<__nv_bfloat16*>(a.y_out), ctx->d_status, a.rows,
                        a.N, a.K, a.rank, a.adapters, a.segments};
  if (moe_knob_value(ctx, "adapter_tiles", tiles_are_quicker(a) ? 1 : 0) != 0 && a.offsets && a.segments > 0)
    return launch_adapter_tiles(ctx, p, stream);
  const int units = units_of(a.rows, a.adapters, a.segments);
  const long long items = (a.rows + kWindow - 1) / kWindow * units;
  const int cluster = cluster_of(a.rows, a.segments, a.offsets != nullptr, a.adapters, a.rank);
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  cfg.gridDim = dim3(static_cast<unsigned>(items * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_of(a.rank, cluster);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(cluster);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  ctx->last_launches += 1;
  auto kernel = a.rank <= 16 ? adapter_rows<2> : a.rank <= 32 ? adapter_rows<4> : a.rank <= 64 ? adapter_rows<8> : adapter_rows<16>;
  return cudaLaunchKernelEx(&cfg, kernel, p, units, cluster) == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

cudaError_t prepare_adapters(moe_ctx* ctx) {
  cudaError_t e = prepare_adapter_tiles(ctx);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(adapter_rows<8>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(64, kMaxCluster));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(adapter_rows<16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(128, kMaxCluster));
  return e;
}

}  // namespace moe
