// Adapters over long segments: tiles of up to 128 rows of one segment on the tensor cores, both products in one launch.
//
// A cluster of up to eight CTAs takes a tile.  First t = x a^T: each CTA has a part of K, x and a come through a TMA ring of 64-deep
// stages; every CTA sends the others their rows of its sums through distributed shared memory, adds the parts of its own rows
// in order, scales them and sends them on as two bf16 terms (16 bits: the error of one term would be that of the output's
// rounding).  Then y += t b^T: each CTA has a range of columns, the terms of t lie in shared memory as the A operand, y and b come
// through TMA rings in tiles of 64 columns, the sum is formed in y's place in shared memory and leaves by TMA.
//
// A tile begins where its segment does or 128 rows later: a TMA box may start at any row.  What a box brings of the rows behind
// the segment's last is computed and not used; tiles of up to 16 rows use boxes of 16.  Segment s has the clusters from
// offsets[s] / 128 + s on, so no list of tiles is built; the rows behind the last segment are one more segment without an adapter.
//
// Warp 0 loads, warp 1 issues the products, warps 2-5 move between accumulator and shared memory; the first of y and b are on
// their way while the parts of t are added.
//
// Bound by HBM in both phases (x in, then y in and out), with a gap of about 8 us between them in which the sums change hands:
// nothing but the first tiles of y is in flight there.  8192 rows in 4 segments, 7168 -> 4096, rank 64: 51.5 us, 5.0 TB/s of the
// 257 MB (39.2 us at the rate of a copy); rank 128: 55 us of kernel.  With scratch for t and two launches it took 62.
#include "adapters.cuh"
#include "ptx_sm100.cuh"
#include "warp_search.cuh"

namespace {

using moe::AdapterParams;

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kTileRows = 128;
constexpr int kShortRows = 16;            // tiles of up to so many rows load that many
constexpr int kSlabRows = 32;
constexpr int kThreads = 192;
constexpr int kBK = 64;                   // values of K in a stage: 128 bytes of bf16
constexpr int kCols = 128;                // accumulator columns: t's, later two tiles of y
constexpr int kXBytes = kTileRows * 128;
constexpr int kMaxStages = 6;
constexpr int kBN = 64;                   // columns of a tile of y
constexpr int kYBytes = kTileRows * 128;
constexpr int kSlabBytes = kYBytes / 4;   // 32 rows of it: what one epilogue warp loads, changes and stores by itself
constexpr int kAtomA = kTileRows * 128;   // 64 ranks of one term of t
constexpr int kAtomB = kBN * 128;         // 64 ranks of b
constexpr int kMaxYStages = 6, kMaxBStages = 4;
constexpr int kMaxCluster = 8;
constexpr int kSumRows = 136;             // a share of the rows from each CTA, rounded up: c ceil(128 / c) for c <= 8

struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], y_full[kMaxYStages][4], b_full[kMaxBStages], b_empty[kMaxBStages], acc_full[2], acc_empty[2],
      sums_full;
  uint32_t tmem;
  int abort_flag;
};

// Shared memory of a CTA: in the second phase the terms of t, b's ring and y's ring; in the first the ring of x and a from the
// start, and behind it the sums that the cluster sends, in the place of y's last tiles; then the barriers.  112 KiB, of which an
// SM holds two, and 224 above 64 ranks.
struct Layout {
  int atoms, rank16, pitch, stage_bytes, stages, y_stages, b_stages, b_at, y_at, sums_at, barriers_at, bytes;
  __host__ __device__ constexpr explicit Layout(int rank)
      : atoms(0), rank16(0), pitch(0), stage_bytes(0), stages(0), y_stages(0), b_stages(0), b_at(0), y_at(0), sums_at(0), barriers_at(0),
        bytes(0) {
    atoms = (rank + 63) / 64;
    rank16 = (rank + 15) / 16 * 16;
    pitch = rank + 4;                                      // floats of a row of sums: an odd number of 16 bytes
    y_stages = atoms == 1 ? 4 : kMaxYStages;
    b_stages = atoms == 1 ? 2 : kMaxBStages;
    b_at = 2 * atoms * kAtomA;
    y_at = b_at + b_stages * atoms * kAtomB;
    barriers_at = y_at + y_stages * kYBytes;               // (the sums leave y's first tile alone: 136 x 132 x 4 < 5 x 16384)
    sums_at = barriers_at - kSumRows * pitch * 4;
    stage_bytes = kXBytes + rank16 * 128;
    stages = sums_at / stage_bytes < kMaxStages ? sums_at / stage_bytes : kMaxStages;
    bytes = barriers_at + static_cast<int>(sizeof(Barriers));
  }
};

static_assert(Layout(128).bytes <= 227 * 1024 && 2 * (Layout(64).bytes + 1024) <= 228 * 1024, "one CTA to an SM, or two");
static_assert(Layout(128).sums_at >= Layout(128).y_at + kYBytes && Layout(64).sums_at >= Layout(64).y_at + kYBytes,
              "the sums leave y's first tile alone");

struct Maps {
  CUtensorMap x, x_short, a, b, in, in_short, out;
};

__device__ __forceinline__ void timed_out(const AdapterParams& p, int where) {
  atomicCAS(&p.status[0], 0, MOE_ERR_TIMEOUT);
  atomicCAS(&p.status[1], 0, 200 + where);
}

// Eight values as two terms of bf16.
__device__ __forceinline__ void two_terms(const float (&v)[8], uint4& hi, uint4& lo) {
  moe::two_terms(v[0], v[1], hi.x, lo.x);
  moe::two_terms(v[2], v[3], hi.y, lo.y);
  moe::two_terms(v[4], v[5], hi.z, lo.z);
  moe::two_terms(v[6], v[7], hi.w, lo.w);
}
// y + d in bf16.
__device__ __forceinline__ uint32_t add_pair(uint32_t y, uint32_t d0, uint32_t d1) {
  return moe::pair(moe::low(y) + __uint_as_float(d0), moe::high(y) + __uint_as_float(d1));
}

// The NaN of a row's `cols` columns formed again: y + t b with t = hi + lo.  `row`, `hi`, `lo`: 128 bytes of a swizzled atom, whose
// 16-byte chunk c lies at c ^ swizzle; b and y begin at the first column.  What is NaN by t, y or b is soon given up (8192 rows of
// 4096 columns, rank 64: 64 us, 73 with all of x NaN, 129 with all of y, 182 with all of b).
__device__ __noinline__ void sum_again(unsigned char* row, const unsigned char* hi, const unsigned char* lo, int swizzle,
                                       const __nv_bfloat16* b, const __nv_bfloat16* y, int cols, int rank) {
  auto terms = [&](int j, float (&t)[8]) {                 // of ranks j to j + 7
    const int at = (j >> 6) * kAtomA + ((((j >> 3) & 7) ^ swizzle) << 4);
    const uint4 h = *reinterpret_cast<const uint4*>(hi + at), l = *reinterpret_cast<const uint4*>(lo + at);
    const uint32_t hs[4] = {h.x, h.y, h.z, h.w}, ls[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      t[2 * q] = moe::low(hs[q]) + moe::low(ls[q]);
      t[2 * q + 1] = moe::high(hs[q]) + moe::high(ls[q]);
    }
  };
  float t[8], all = 0.f;
  for (int j = 0; j < rank; j += 8) {
    terms(j, t);
#pragma unroll
    for (int q = 0; q < 8; ++q) all += fabsf(t[q]);
  }
  if (all != all) return;                                  // t has a NaN, and so has every column
  for (int n = 0; n < cols; n += 8) {
    uint4* at = reinterpret_cast<uint4*>(row + (((n >> 3) ^ swizzle) << 4));
    uint4 sum = *at;
    if (!moe::has_nan(moe::largest(moe::largest(sum.x, sum.y, sum.z), sum.w, sum.w))) continue;
    const uint4 old = *reinterpret_cast<const uint4*>(y + n);
    const uint32_t was[4] = {old.x, old.y, old.z, old.w}, now[4] = {sum.x, sum.y, sum.z, sum.w};
    float d[8];                                            // NaN where nothing is to be found
    bool some = false;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float y0 = c & 1 ? moe::high(was[c / 2]) : moe::low(was[c / 2]), s0 = c & 1 ? moe::high(now[c / 2]) : moe::low(now[c / 2]);
      d[c] = s0 != s0 && y0 == y0 ? 0.f : __uint_as_float(0x7FC00000u);
      some |= d[c] == d[c];
    }
    for (int j = 0; j < rank && some; j += 8) {
      terms(j, t);
      uint4 w[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) w[c] = __ldg(reinterpret_cast<const uint4*>(b + static_cast<size_t>(n + c) * rank + j));
      some = false;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t ws[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) d[c] = fmaf(t[2 * q + 1], moe::high(ws[q]), fmaf(t[2 * q], moe::low(ws[q]), d[c]));
        some |= d[c] == d[c];
      }
    }
    uint32_t v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float s0 = moe::low(now[q]), s1 = moe::high(now[q]);
      v[q] = moe::pair(s0 == s0 ? s0 : moe::low(was[q]) + d[2 * q], s1 == s1 ? s1 : moe::high(was[q]) + d[2 * q + 1]);
    }
    *at = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

// Grid: a cluster of `cluster` CTAs per tile.
__global__ void __launch_bounds__(kThreads)
adapter_tiles(const __grid_constant__ Maps maps, const AdapterParams p, int cluster) {
  extern __shared__ __align__(1024) unsigned char base[];
  const Layout lay(p.rank);
  Barriers& bar = *reinterpret_cast<Barriers*>(base + lay.barriers_at);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3;
  const int tile = blockIdx.x / cluster, part = blockIdx.x - tile * cluster;

  // Tensor memory first: the SM takes its second CTA only when the first has given up the right to allocate (with the search in
  // front of it, half of the CTAs began 2.4 us later).
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(&bar.tmem), kCols);
    ptx::tmem_relinquish();
    ptx::tc_fence_before_sync();
    __syncwarp();
  }
  auto leave = [&]() {
    if (warp == 1) ptx::tmem_dealloc(*static_cast<volatile uint32_t*>(&bar.tmem), kCols);
  };
  if (threadIdx.x == 0) {
    ptx::prefetch_tensormap(&maps.x);
    ptx::prefetch_tensormap(&maps.a);
  }
  // the tile's segment, rows and adapter: each warp finds them by itself
  auto bound = [&](int s) {
    const long long o = __ldg(p.offsets + s);
    return o < 0 ? 0LL : o > p.rows ? p.rows : o;
  };
  const int seg = moe::last_at_or_below(p.segments + 1, tile, lane, [&](int s) { return bound(s) / kTileRows + s; });
  if (seg < 0) return leave();
  const long long begin = bound(seg), end = seg < p.segments ? bound(seg + 1) : p.rows;
  const long long row0 = begin + (tile - (begin / kTileRows + seg)) * kTileRows;
  if (row0 < begin || row0 >= end) return leave();         // (the whole cluster; below begin: offsets that do not ascend)
  const int m = static_cast<int>(end - row0 < kTileRows ? end - row0 : kTileRows);
  int id = seg < p.segments ? __ldg(p.adapter_of + seg) : -1;
  if (id >= p.adapters) {
    if (part == 0 && threadIdx.x == 0) {
      atomicCAS(&p.status[0], 0, MOE_ERR_BAD_ROUTING);
      atomicCAS(&p.status[1], 0, seg);
    }
    id = -1;
  }
  const bool has = id >= 0;
  if (!has && p.y_in == p.y_out) return leave();           // nothing to add and nothing to copy

  const uint32_t base_at = ptx::smem_u32(base);
  const int blocks = (p.K + kBK - 1) / kBK, parts = min(cluster, blocks);
  const bool sums = has && part < parts;                   // this CTA has a part of K
  // (every parts-th block of K: the cluster reads neighbouring lines of x at a time)
  const int tiles = (p.N - 1) / kBN + 1;
  const int n0 = static_cast<int>(static_cast<long long>(tiles) * part / cluster);
  const int n1 = static_cast<int>(static_cast<long long>(tiles) * (part + 1) / cluster);
  const int y_ahead = min(lay.y_stages, n1 - n0);
  const bool few = m <= kShortRows;
  const CUtensorMap* tm_x = few ? &maps.x_short : &maps.x;
  const uint32_t x_bytes = few ? kShortRows * 128 : kXBytes;                 // of x in a stage
  if (threadIdx.x == 0) {
    for (int i = 0; i < lay.stages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.empty[i]), 1);
    }
    for (int i = 0; i < lay.y_stages; ++i)
      for (int w = 0; w < 4; ++w) ptx::mbar_init(ptx::smem_u32(&bar.y_full[i][w]), 1);
    for (int i = 0; i < lay.b_stages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.b_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.b_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.acc_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.acc_empty[i]), 4);
    }
    ptx::mbar_init(ptx::smem_u32(&bar.sums_full), 1);
    bar.abort_flag = 0;
    ptx::fence_barrier_init();
  }
  __syncthreads();
  if (has) ptx::cluster_arrive();                          // (waited for before anything is sent: every CTA has begun)
  ptx::tc_fence_after_sync();
  const uint32_t tmem = bar.tmem, lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
  volatile int* abort_flag = &bar.abort_flag;
  const int r = quarter * 32 + lane;                       // the row of an epilogue thread
  int y_issued = 0, b_issued = 0;                          // (warp 0's lane 0)
  const uint64_t once = ptx::l2_policy_evict_first();      // x and y are read once: b, a and y's writes may stay in L2 (51.5 us; 57.5 without)
  auto load_y = [&](int slot, int n, int w) {              // rows 32 w and on
    if (32 * w >= m) return;
    const uint32_t full = ptx::smem_u32(&bar.y_full[slot][w]);
    ptx::mbar_expect_tx(full, few ? kShortRows * 128 : kSlabBytes);
    ptx::tma_load_2d_hint(base_at + lay.y_at + slot * kYBytes + w * kSlabBytes, few ? &maps.in_short : &maps.in, full, n * kBN,
                          static_cast<int>(row0) + 32 * w, once);
  };
  auto load_b = [&](int slot, int n) {
    const uint32_t full = ptx::smem_u32(&bar.b_full[slot]);
    ptx::mbar_expect_tx(full, lay.atoms * kAtomB);
    for (int k = 0; k < lay.atoms; ++k)
      ptx::tma_load_2d(base_at + lay.b_at + (slot * lay.atoms + k) * kAtomB, &maps.b, full, k * 64, id * p.N + n * kBN);
  };

  // ------------------------------------------------------------------------------------------------ t = x a^T
  if (has) {
    const int share = (m + cluster - 1) / cluster;         // rows of a CTA, at most
    if (warp == 0) {
      if (lane == 0 && sums) {
        int stage = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int kb = part; kb < blocks; kb += parts) {
          ok = ptx::mbar_wait(ptx::smem_u32(&bar.empty[stage]), phase, abort_flag);
          if (!ok) break;
          const uint32_t full = ptx::smem_u32(&bar.full[stage]), at = base_at + stage * lay.stage_bytes;
          ptx::mbar_expect_tx(full, x_bytes + lay.rank16 * 128);
          ptx::tma_load_2d_hint(at, tm_x, full, kb * kBK, static_cast<int>(row0), once);
          ptx::tma_load_2d(at + kXBytes, &maps.a, full, kb * kBK, id * p.rank);
          if (++stage == lay.stages) { stage = 0; phase ^= 1u; }
        }
        ok = ok && ptx::mbar_wait(ptx::smem_u32(&bar.sums_full), 0, abort_flag);
        if (!ok) timed_out(p, 1);
      }
      // nothing reads the ring any more: b, and y's tiles in front of the sums, may come
      if (lane == 0 && !*abort_flag) {
        for (; b_issued < min(lay.b_stages, n1 - n0); ++b_issued) load_b(b_issued, n0 + b_issued);
        for (; y_issued < y_ahead && lay.y_at + (y_issued + 1) * kYBytes <= lay.sums_at; ++y_issued)
          for (int w = 0; w < 4; ++w) load_y(y_issued, n0 + y_issued, w);
      }
      __syncwarp();
      ptx::cluster_wait();
    } else if (warp == 1) {
      if (sums) {
        // (the whole warp runs the loop, one lane issues: the descriptors stay warp-uniform)
        const uint32_t idesc = ptx::idesc_bf16_f32(kTileRows, lay.rank16);
        const uint64_t a0 = ptx::smem_desc_sw128(base_at);
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = part; kb < blocks; kb += parts) {
          ptx::mbar_wait_or_flag(ptx::smem_u32(&bar.full[stage]), phase, abort_flag, 2);
          ptx::tc_fence_after_sync();
          if (ptx::elect_one()) {
            const uint64_t a = a0 + static_cast<uint32_t>(stage * lay.stage_bytes) / 16, b = a + kXBytes / 16;
#pragma unroll
            for (int k = 0; k < kBK / 16; ++k) ptx::tc_mma_bf16(tmem, a + 2 * k, b + 2 * k, idesc, kb > part || k > 0);
            ptx::tc_commit(ptx::smem_u32(&bar.empty[stage]));
          }
          __syncwarp();
          if (++stage == lay.stages) { stage = 0; phase ^= 1u; }
        }
        if (ptx::elect_one()) ptx::tc_commit(ptx::smem_u32(&bar.sums_full));
        if (*abort_flag && lane == 0) timed_out(p, 2);
      }
      __syncwarp();
      ptx::cluster_wait();
    } else {
      const bool ok = !sums || __all_sync(kFull, ptx::mbar_wait(ptx::smem_u32(&bar.sums_full), 0, abort_flag));
      __syncwarp();
      ptx::cluster_wait();
      if (!ok && lane == 0) timed_out(p, 3);
      if (ok && sums && quarter * 32 < m) {
        ptx::tc_fence_after_sync();
        // row r goes to the CTA in whose share it lies: the last q with m q / cluster <= r
        const int owner = ((r + 1) * cluster + m - 1) / m - 1, first = m * owner / cluster;
        const uint32_t dst = ptx::map_to_cta(base_at + lay.sums_at + (part * share + r - first) * lay.pitch * 4, min(owner, cluster - 1));
        for (int j = 0; j < p.rank; j += 32) {             // (columns behind the rank hold something, or nothing yet)
          uint32_t v[32];
          ptx::tmem_ld_32x32(lanes + j, v);
          ptx::tmem_ld_wait();
          if (r < m) {
#pragma unroll
            for (int q = 0; q < 32; q += 4)
              if (j + q < p.rank) moe::st_cluster(dst + (j + q) * 4, make_uint4(v[q], v[q + 1], v[q + 2], v[q + 3]));
          }
        }
        ptx::tc_fence_before_sync();
      }
    }
    __syncwarp();
    ptx::cluster_sync();
    ptx::tc_fence_after_sync();
    // this CTA's rows: the parts of K in order, and the terms to every CTA; eight ranks a step
    const float f = p.scale != nullptr ? __ldg(p.scale + id) : 1.f;
    const int r0 = m * part / cluster, r1 = m * (part + 1) / cluster, chunks = lay.rank16 / 8;
    for (int i = threadIdx.x; i < (r1 - r0) * chunks; i += kThreads) {
      const int local = i / chunks, row = r0 + local, j = i - local * chunks;
      uint4 hi = make_uint4(0u, 0u, 0u, 0u), lo = hi;      // (up to whole steps of the product: zeros)
      if (8 * j < p.rank) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const float* src = reinterpret_cast<const float*>(base + lay.sums_at) + local * lay.pitch + 8 * j;
#pragma unroll
        for (int s = 0; s < kMaxCluster; ++s) {
          if (s < parts) {
            const float4 a = *reinterpret_cast<const float4*>(src + s * share * lay.pitch);
            const float4 b = *reinterpret_cast<const float4*>(src + s * share * lay.pitch + 4);
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
            v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
          }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] *= f;
        two_terms(v, hi, lo);
      }
      const uint32_t at = base_at + (j >> 3) * kAtomA + row * 128 + (((j & 7) ^ (row & 7)) << 4);
#pragma unroll
      for (int q = 0; q < kMaxCluster; ++q) {
        if (q < cluster) {
          const uint32_t to = ptx::map_to_cta(at, q);
          moe::st_cluster(to, hi);
          moe::st_cluster(to + lay.atoms * kAtomA, lo);
        }
      }
    }
    // the terms are read by the products, and the sums' place belongs to TMA again
    __syncwarp();
    ptx::fence_proxy_async_all();
    ptx::cluster_sync();
  }

  // ------------------------------------------------------------------------------------------------ y += t b^T
  if (warp == 0) {
    if (lane == 0) {
      bool ok = true;
      for (; y_issued < y_ahead; ++y_issued)
        for (int w = 0; w < 4; ++w) load_y(y_issued, n0 + y_issued, w);
      int bs = 0;
      uint32_t b_phase = 1;
      for (int i = n0; i < n1 && has; ++i) {
        if (i - n0 >= b_issued) {
          ok = ptx::mbar_wait(ptx::smem_u32(&bar.b_empty[bs]), b_phase, abort_flag);
          if (!ok) break;
          load_b(bs, i);
        }
        if (++bs == lay.b_stages) { bs = 0; b_phase ^= 1u; }
      }
      if (!ok) timed_out(p, 4);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (has) {
      const uint32_t idesc = ptx::idesc_bf16_f32(kTileRows, kBN);
      const uint64_t a0 = ptx::smem_desc_sw128(base_at), b0 = ptx::smem_desc_sw128(base_at + lay.b_at);
      const int steps = lay.rank16 / 16;
      int bs = 0, acc = 0;
      uint32_t b_phase = 0, acc_phase = 1;
      ptx::fence_proxy_async_all();
      for (int i = n0; i < n1; ++i) {
        ptx::mbar_wait_or_flag(ptx::smem_u32(&bar.b_full[bs]), b_phase, abort_flag, 5);
        ptx::mbar_wait_or_flag(ptx::smem_u32(&bar.acc_empty[acc]), acc_phase, abort_flag, 5);
        ptx::tc_fence_after_sync();
        if (ptx::elect_one()) {
          const uint32_t d = tmem + acc * kBN;
          const uint64_t b = b0 + static_cast<uint32_t>(bs * lay.atoms * kAtomB) / 16;
#pragma unroll
          for (int k = 0; k < 8; ++k) {                    // both terms of 16 ranks on the same 16 of b
            if (k < steps) {
              const uint64_t at = a0 + (k >> 2) * (kAtomA / 16) + 2 * (k & 3), with = b + (k >> 2) * (kAtomB / 16) + 2 * (k & 3);
              ptx::tc_mma_bf16(d, at, with, idesc, k > 0);
              ptx::tc_mma_bf16(d, at + lay.atoms * (kAtomA / 16), with, idesc, 1);
            }
          }
          ptx::tc_commit(ptx::smem_u32(&bar.b_empty[bs]));
          ptx::tc_commit(ptx::smem_u32(&bar.acc_full[acc]));
        }
        __syncwarp();
        if (++bs == lay.b_stages) { bs = 0; b_phase ^= 1u; }
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (*abort_flag && lane == 0) timed_out(p, 5);
    }
    __syncwarp();
  } else {
    const bool whole = quarter * 32 + 32 <= m, live = quarter * 32 < m;      // the warp's rows: all of them, any of them
    int ys = 0, acc = 0;
    uint32_t y_phase = 0, acc_phase = 0;
    for (int i = n0; i < n1; ++i) {
      const bool ok =
          __all_sync(kFull, (!live || ptx::mbar_wait(ptx::smem_u32(&bar.y_full[ys][quarter]), y_phase, abort_flag)) &&
                                (!has || ptx::mbar_wait(ptx::smem_u32(&bar.acc_full[acc]), acc_phase, abort_flag)));
      if (!ok) {
        if (lane == 0) timed_out(p, 6);
        break;
      }
      unsigned char* slab = base + lay.y_at + ys * kYBytes + quarter * kSlabBytes;
      if (live && has) {
        unsigned char* row = slab + lane * 128;
        ptx::tc_fence_after_sync();
        uint32_t v[32], w[32];
        ptx::tmem_ld_32x32(lanes + acc * kBN, v);
        ptx::tmem_ld_32x32(lanes + acc * kBN + 32, w);
        uint4 y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] = *reinterpret_cast<const uint4*>(row + ((c ^ (lane & 7)) << 4));
        ptx::tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const uint32_t* d = c < 4 ? v + 8 * c : w + 8 * (c - 4);
          y[c] = make_uint4(add_pair(y[c].x, d[0], d[1]), add_pair(y[c].y, d[2], d[3]), add_pair(y[c].z, d[4], d[5]),
                            add_pair(y[c].w, d[6], d[7]));
          *reinterpret_cast<uint4*>(row + ((c ^ (lane & 7)) << 4)) = y[c];
        }
        uint32_t most[4] = {y[0].x, y[0].y, y[0].z, y[0].w};
#pragma unroll
        for (int c = 1; c < 7; c += 2) {
          most[0] = moe::largest(most[0], y[c].x, y[c + 1].x);
          most[1] = moe::largest(most[1], y[c].y, y[c + 1].y);
          most[2] = moe::largest(most[2], y[c].z, y[c + 1].z);
          most[3] = moe::largest(most[3], y[c].w, y[c + 1].w);
        }
        const uint32_t nan = moe::largest(moe::largest(most[0], most[1], y[7].x), moe::largest(most[2], most[3], y[7].y),
                                          moe::largest(y[7].z, y[7].w, y[7].w));
        if (r < m && moe::has_nan(nan))
          // (y as it was: what leaves goes by this warp, later)
          sum_again(row, base + r * 128, base + r * 128 + lay.atoms * kAtomA, lane & 7,
                    p.b + (static_cast<size_t>(id) * p.N + i * kBN) * p.rank, p.y_in + static_cast<size_t>(row0 + r) * p.N + i * kBN,
                    min(kBN, p.N - i * kBN), p.rank);
        ptx::tc_fence_before_sync();
      }
      if (whole) ptx::fence_proxy_async_smem();
      __syncwarp();
      if (has) {
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&bar.acc_empty[acc]));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (live && !whole) {                                // all 32 rows leave by TMA, the rows of a segment's end from here
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          const int rr = it * 4 + (lane >> 3), c = lane & 7;
          if (quarter * 32 + rr < m && i * kBN + 8 * c < p.N)
            *reinterpret_cast<uint4*>(p.y_out + static_cast<size_t>(row0 + quarter * 32 + rr) * p.N + i * kBN + 8 * c) =
                *reinterpret_cast<const uint4*>(slab + rr * 128 + ((c ^ (rr & 7)) << 4));
        }
        ptx::fence_proxy_async_smem();                     // TMA writes the slab next: behind these writes and reads
        __syncwarp();
      }
      if (lane == 0) {
        if (whole) {
          ptx::tma_store_2d(&maps.out, base_at + lay.y_at + ys * kYBytes + quarter * kSlabBytes, i * kBN,
                            static_cast<int>(row0) + quarter * 32);
          ptx::bulk_commit_group();
        }
        if (i > n0 && i - 1 + y_ahead < n1) {              // the rows before these have left: later ones take their place
          ptx::bulk_wait_group_read_but_one();
          load_y(ys == 0 ? lay.y_stages - 1 : ys - 1, i - 1 + y_ahead, quarter);
        }
      }
      if (++ys == lay.y_stages) { ys = 0; y_phase ^= 1u; }
    }
    if (lane == 0) ptx::bulk_wait_group_read_all();
    __syncwarp();
  }

  // Frees what the CTA holds; after a wait that gave up, copies in flight get time to land first.
  __syncthreads();
  if (bar.abort_flag) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, kCols);
  }
}

bool encode(moe_ctx* ctx, CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows) {
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {cols * 2};
  const cuuint32_t box[2] = {64u, box_rows};
  const cuuint32_t elem[2] = {1u, 1u};
  return ctx->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, elem,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

long long tiles_of(long long rows, int segments) { return rows / kTileRows + segments + 1; }

// CTAs of a tile: as many as are resident at once (two on an SM, one above 64 ranks), at most a portable cluster.  8192 rows, rank 64:
// 51.5 us; 71.8 with one CTA to an SM.  8192 rows, rank 128: 69.9 us from one kernel to the next; 103 with clusters for two.
int cluster_of(const moe_ctx* ctx, long long tiles, int rank, int N, int K) {
  const int most = (N - 1) / kBN + 1 > (K - 1) / kBK + 1 ? (N - 1) / kBN + 1 : (K - 1) / kBK + 1;
  long long c = (rank > 64 ? 1LL : 2LL) * ctx->num_sms / tiles;
  if (c > kMaxCluster) c = kMaxCluster;
  if (c > most) c = most;
  return c < 1 ? 1 : static_cast<int>(c);
}

}  // namespace

namespace moe {

moe_status launch_adapter_tiles(moe_ctx* ctx, const AdapterParams& p, cudaStream_t stream) {
  Maps m;
  const uint64_t factor_rows = static_cast<uint64_t>(p.adapters) * p.rank, out_rows = static_cast<uint64_t>(p.adapters) * p.N;
  if (!encode(ctx, &m.x, p.x, p.rows, p.K, kTileRows) || !encode(ctx, &m.x_short, p.x, p.rows, p.K, kShortRows) ||
      !encode(ctx, &m.a, p.a, factor_rows, p.K, Layout(p.rank).rank16) ||
      !encode(ctx, &m.b, p.b, out_rows, p.rank, kBN) || !encode(ctx, &m.in, p.y_in, p.rows, p.N, kSlabRows) ||
      !encode(ctx, &m.in_short, p.y_in, p.rows, p.N, kShortRows) || !encode(ctx, &m.out, p.y_out, p.rows, p.N, kSlabRows))
    return MOE_ERR_CUDA;
  const long long tiles = tiles_of(p.rows, p.segments);
  const int cluster = cluster_of(ctx, tiles, p.rank, p.N, p.K);
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Layout(p.rank).bytes;
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(cluster);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  ctx->last_launches += 1;
  return cudaLaunchKernelEx(&cfg, adapter_tiles, m, p, cluster) == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

cudaError_t prepare_adapter_tiles(moe_ctx* ctx) {
  (void)ctx;
  return cudaFuncSetAttribute(adapter_tiles, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout(128).bytes);
}

}  // namespace moe
