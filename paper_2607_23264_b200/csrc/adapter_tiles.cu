// Adapters over long segments: tiles of 128 rows on the tensor cores.
//
// A tile's rows may belong to several adapters.  Neither product masks anything: an adapter's columns of the accumulator are
// computed for all 128 rows, and a row takes those of its own adapter.
//
// adapter_shrink_tiles : t = x a^T, a CTA per tile and part of K.  x and the factors of the tile's adapters (up to 128 columns of the
//                        accumulator in a pass) come through a TMA ring of 64-deep stages; warp 0 loads, warp 1 issues the
//                        products, warps 2-5 write each row's part of t to the scratch, one fp32 copy per part of K.
// adapter_expand_tiles : y += t b^T, a CTA per tile and range of columns.  t is summed over the parts of K, scaled, and cut into two bf16
//                        terms (16 bits; the error of one term would be that of the output's rounding) that stay in shared
//                        memory as the A operand; y and b come through TMA rings in tiles of 64 columns, the sum is formed in
//                        y's place in shared memory and leaves by TMA.  Rows without an adapter pass through untouched.  Starts
//                        while the first kernel runs (programmatic launch): its loads do not depend on t.
#include "adapters.cuh"
#include "ptx_sm100.cuh"

namespace {

using moe::AdapterParams;

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kTileRows = 128;
constexpr int kThreads = 192;             // TMA, MMA and four epilogue warps
constexpr int kBK = 64;                   // values of K in a stage: 128 bytes of bf16
constexpr int kCols = 128;                // accumulator columns of a shrink pass, and both accumulators of the expansion
constexpr int kXBytes = kTileRows * 128;
constexpr int kStageBytes = kXBytes + kCols * 128;
constexpr int kMaxStages = 6;
constexpr int kBN = 64;                   // columns of an expand tile
constexpr int kYBytes = kTileRows * 128;
constexpr int kAtomA = kTileRows * 128;   // 64 ranks of one term of t
constexpr int kAtomB = kBN * 128;         // 64 ranks of b
constexpr int kYStages = 3, kBStages = 3;
constexpr int kCachedOffsets = 513;
constexpr int kMaxSplits = 8;            // CTAs of a cluster

struct alignas(16) TileIds {
  int id[kTileRows];                      // adapter of each row, -1 without one
  int slot[kTileRows];                    // its place in `list`
  int list[kTileRows];                    // the tile's adapters in order of their first row
  int place[kTileRows];
  int warp_count[4];
  int32_t offsets[kCachedOffsets];
};
struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], y_full[kYStages], acc_full[2], acc_empty[2], t_full;
  uint32_t tmem;
  int abort_flag;
};

__device__ __forceinline__ void timed_out(const AdapterParams& p, int where) {
  atomicCAS(&p.status[0], 0, MOE_ERR_TIMEOUT);
  atomicCAS(&p.status[1], 0, 200 + where);
}

// Fills `s` for the tile at row0; by the whole CTA.  Returns the number of adapters.
__device__ int collect(const AdapterParams& p, long long row0, TileIds* s, bool report) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t* offsets = p.offsets;
  if (offsets != nullptr && p.segments < kCachedOffsets) {
    for (int i = tid; i <= p.segments; i += kThreads) s->offsets[i] = __ldg(offsets + i);
    offsets = s->offsets;
  }
  __syncthreads();
  if (tid < kTileRows) s->id[tid] = moe::adapter_of_row(p, offsets, row0 + tid, report);
  __syncthreads();
  int id = -1, first = tid;
  unsigned leaders = 0;
  if (tid < kTileRows) {
    id = s->id[tid];
    first = warp * 32 + __ffs(__match_any_sync(kFull, id)) - 1;
    const int4* rows = reinterpret_cast<const int4*>(s->id);
    for (int r = 8 * warp - 1; r >= 0; --r) {              // earlier warps' rows, the lowest last
      const int4 v = rows[r];
      if (v.w == id) first = 4 * r + 3;
      if (v.z == id) first = 4 * r + 2;
      if (v.y == id) first = 4 * r + 1;
      if (v.x == id) first = 4 * r;
    }
    leaders = __ballot_sync(kFull, id >= 0 && first == tid);
    if (lane == 0) s->warp_count[warp] = __popc(leaders);
  }
  __syncthreads();
  int total = 0;
  if (tid < kTileRows && id >= 0 && first == tid) {
    int at = __popc(leaders & ((1u << lane) - 1));
    for (int w = 0; w < warp; ++w) at += s->warp_count[w];
    s->list[at] = id;
    s->place[tid] = at;
  }
  for (int w = 0; w < 4; ++w) total += s->warp_count[w];
  __syncthreads();
  if (tid < kTileRows) s->slot[tid] = id >= 0 ? s->place[first] : -1;
  __syncthreads();
  return total;
}

// Frees what the CTA holds; after a wait that gave up, copies in flight get time to land first.
__device__ __forceinline__ void finish(Barriers* bar, int warp) {
  __syncthreads();
  if (bar->abort_flag) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(bar->tmem, kCols);
  }
}

// Eight values as two terms of bf16: v - hi is exact, so hi + lo keeps 16 bits.
__device__ __forceinline__ uint32_t pair(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ void two_terms(const float (&v)[8], uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = pair(v[2 * i], v[2 * i + 1]);
    // (an infinite or NaN value: the first term says it all)
    const float a = v[2 * i] - low(h[i]), b = v[2 * i + 1] - high(h[i]);
    l[i] = pair(a == a ? a : 0.f, b == b ? b : 0.f);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// Grid: a cluster of p.splits CTAs per tile.
__global__ void __launch_bounds__(kThreads)
adapter_shrink_tiles(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_a, const AdapterParams p,
                     int stages, int rank16) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ TileIds ids;
  __shared__ Barriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile = blockIdx.x / p.splits, split = blockIdx.x - tile * p.splits;
  const long long row0 = static_cast<long long>(tile) * kTileRows;
  unsigned char* base = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t ring = ptx::smem_u32(base);
  const int blocks = (p.K + kBK - 1) / kBK;
  const int kb0 = static_cast<int>(static_cast<long long>(blocks) * split / p.splits);
  const int kb1 = static_cast<int>(static_cast<long long>(blocks) * (split + 1) / p.splits);
  const int ahead = min(stages, kb1 - kb0);                // stages whose x is on its way before the adapters are known
  ptx::launch_dependents();
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.full[i]), 2);      // x and the factors report on their own
      ptx::mbar_init(ptx::smem_u32(&bar.empty[i]), 1);
    }
    ptx::mbar_init(ptx::smem_u32(&bar.acc_full[0]), 1);
    bar.abort_flag = 0;
    ptx::fence_barrier_init();
    for (int i = 0; i < ahead; ++i) {
      ptx::mbar_expect_tx(ptx::smem_u32(&bar.full[i]), kXBytes);
      ptx::tma_load_2d(ring + i * kStageBytes, &tm_x, ptx::smem_u32(&bar.full[i]), (kb0 + i) * kBK, static_cast<int>(row0));
    }
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(&bar.tmem), kCols);
    ptx::tmem_relinquish();
    ptx::tc_fence_before_sync();
  }
  const int count = collect(p, row0, &ids, split == 0);    // (its barriers order the initialisation above as well)
  ptx::tc_fence_after_sync();
  const uint32_t tmem = bar.tmem;
  volatile int* abort_flag = &bar.abort_flag;
  const int per_round = kCols / rank16;                    // adapters
  const int pitch = p.rank + 4;                            // floats of a row of the exchanged sums: an odd number of 16 bytes

  int stage = 0;
  uint32_t phase = warp == 0 ? 1 : 0;
  for (int s0 = 0, round = 0; s0 < count; s0 += per_round, ++round) {
    const int n = min(per_round, count - s0);
    if (warp == 0) {
      if (lane == 0) {
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!ptx::mbar_wait(ptx::smem_u32(&bar.empty[stage]), phase, abort_flag)) {
            timed_out(p, 1);
            break;
          }
          const uint32_t full = ptx::smem_u32(&bar.full[stage]), at = ring + stage * kStageBytes;
          if (round > 0 || kb >= kb0 + ahead) {
            ptx::mbar_expect_tx(full, kXBytes);
            ptx::tma_load_2d(at, &tm_x, full, kb * kBK, static_cast<int>(row0));
          }
          ptx::mbar_expect_tx(full, n * rank16 * 128);
          for (int i = 0; i < n; ++i)
            ptx::tma_load_2d(at + kXBytes + i * rank16 * 128, &tm_a, full, kb * kBK, ids.list[s0 + i] * p.rank);
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      if (lane == 0) {
        const uint32_t idesc = ptx::idesc_bf16_f32(kTileRows, n * rank16);
        bool ok = true;
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = ptx::mbar_wait(ptx::smem_u32(&bar.full[stage]), phase, abort_flag);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const uint32_t at = ring + stage * kStageBytes;
          const uint64_t a = ptx::smem_desc_sw128(at), b = ptx::smem_desc_sw128(at + kXBytes);
#pragma unroll
          for (int k = 0; k < kBK / 16; ++k) ptx::tc_mma_bf16(tmem, a + 2 * k, b + 2 * k, idesc, kb > kb0 || k > 0);
          ptx::tc_commit(ptx::smem_u32(&bar.empty[stage]));
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
        if (ok) ptx::tc_commit(ptx::smem_u32(&bar.acc_full[0]));
        else timed_out(p, 2);
      }
      __syncwarp();
    } else {
      // each row's sums into the ring's place: every stage has been consumed when the accumulator is complete
      const int quarter = warp & 3, r = quarter * 32 + lane, slot = ids.slot[r];
      const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
      if (!__all_sync(kFull, ptx::mbar_wait(ptx::smem_u32(&bar.acc_full[0]), round & 1, abort_flag))) {
        if (lane == 0) timed_out(p, 3);
      } else {
        ptx::tc_fence_after_sync();
        float* dst = reinterpret_cast<float*>(base) + r * pitch;
        for (int i = 0; i < n; ++i) {
          const bool mine = slot == s0 + i;
          if (!__any_sync(kFull, mine)) continue;
          for (int j = 0; j < p.rank; j += 8) {
            uint32_t v[8];
            ptx::tmem_ld_32x8(lanes + i * rank16 + j, v);
            ptx::tmem_ld_wait();
            if (mine) {
              *reinterpret_cast<uint4*>(dst + j) = make_uint4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<uint4*>(dst + j + 4) = make_uint4(v[4], v[5], v[6], v[7]);
            }
          }
        }
        ptx::tc_fence_before_sync();
      }
    }
    // the cluster's sums over its parts of K, a share of the rows per CTA; two terms of bf16
    ptx::cluster_sync();
    ptx::tc_fence_after_sync();
    const int r0 = kTileRows * split / p.splits, r1 = kTileRows * (split + 1) / p.splits, chunks = p.rank / 8;
    for (int i = threadIdx.x; i < (r1 - r0) * chunks; i += kThreads) {
      const int r = r0 + i / chunks, j = 8 * (i % chunks), slot = ids.slot[r];
      if (slot < s0 || slot >= s0 + n) continue;
      const uint32_t at = ring + (r * pitch + j) * 4;
      float4 a[kMaxSplits], b[kMaxSplits];
#pragma unroll
      for (int s = 0; s < kMaxSplits; ++s) {
        a[s] = b[s] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s < p.splits) {
          const uint32_t from = ptx::map_to_cta(at, s);
          a[s] = ptx::ld_cluster_f4(from);
          b[s] = ptx::ld_cluster_f4(from + 16);
        }
      }
      float v[8] = {a[0].x, a[0].y, a[0].z, a[0].w, b[0].x, b[0].y, b[0].z, b[0].w};
#pragma unroll
      for (int s = 1; s < kMaxSplits; ++s) {
        if (s < p.splits) {
          v[0] += a[s].x; v[1] += a[s].y; v[2] += a[s].z; v[3] += a[s].w;
          v[4] += b[s].x; v[5] += b[s].y; v[6] += b[s].z; v[7] += b[s].w;
        }
      }
      if (p.scale != nullptr) {
        const float f = __ldg(p.scale + ids.id[r]);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] *= f;
      }
      uint4 hi, lo;
      two_terms(v, hi, lo);
      __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(p.t) + (row0 + r) * p.rank + j;
      *reinterpret_cast<uint4*>(to) = hi;
      *reinterpret_cast<uint4*>(to + static_cast<size_t>(p.rows) * p.rank) = lo;
    }
    ptx::fence_proxy_async_smem();                         // the sums' place becomes the ring again
    ptx::cluster_sync();
  }
  if (count == 0 && threadIdx.x == 0) {                    // nothing asks for the x on its way: it lands first
    for (int i = 0; i < ahead; ++i) {
      ptx::mbar_arrive(ptx::smem_u32(&bar.full[i]));
      ptx::mbar_wait(ptx::smem_u32(&bar.full[i]), 0, abort_flag);
    }
  }
  finish(&bar, warp);
}

// The four epilogue warps meet; whether any of them has given up.
__device__ __forceinline__ bool epilogue_meets(bool gave_up) {
  uint32_t any;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.b32 p, %1, 0;\n"
      "barrier.cta.red.or.pred q, 2, 128, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(any)
      : "r"(static_cast<uint32_t>(gave_up))
      : "memory");
  return any != 0;
}

__global__ void __launch_bounds__(kThreads)
adapter_expand_tiles(const __grid_constant__ CUtensorMap tm_t, const __grid_constant__ CUtensorMap tm_b,
                     const __grid_constant__ CUtensorMap tm_in, const __grid_constant__ CUtensorMap tm_out,
                     const AdapterParams p, int groups) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ TileIds ids;
  __shared__ Barriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile = blockIdx.x / groups, group = blockIdx.x - tile * groups;
  const long long row0 = static_cast<long long>(tile) * kTileRows;
  const int atoms = (p.rank + 63) / 64;
  unsigned char* base = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* ybase = base + 2 * atoms * kAtomA;        // A: the atoms of the first terms, then of the second
  const uint32_t a_at = ptx::smem_u32(base), y_at = ptx::smem_u32(ybase), b_at = y_at + kYStages * kYBytes;
  const int tiles = (p.N - 1) / kBN + 1;
  const int n0 = static_cast<int>(static_cast<long long>(tiles) * group / groups);
  const int n1 = static_cast<int>(static_cast<long long>(tiles) * (group + 1) / groups);
  const int ahead = min(kYStages, n1 - n0);                // tiles of y on their way before the adapters are known
  if (threadIdx.x == 0) {
    for (int i = 0; i < kBStages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.empty[i]), 1);
    }
    for (int i = 0; i < kYStages; ++i) ptx::mbar_init(ptx::smem_u32(&bar.y_full[i]), 1);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.acc_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.acc_empty[i]), 4);
    }
    ptx::mbar_init(ptx::smem_u32(&bar.t_full), 1);
    bar.abort_flag = 0;
    ptx::fence_barrier_init();
    for (int i = 0; i < ahead; ++i) {
      ptx::mbar_expect_tx(ptx::smem_u32(&bar.y_full[i]), kYBytes);
      ptx::tma_load_2d(y_at + i * kYBytes, &tm_in, ptx::smem_u32(&bar.y_full[i]), (n0 + i) * kBN, static_cast<int>(row0));
    }
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(&bar.tmem), kCols);
    ptx::tmem_relinquish();
    ptx::tc_fence_before_sync();
  }
  const int count = collect(p, row0, &ids, false);
  ptx::tc_fence_after_sync();
  const uint32_t tmem = bar.tmem;
  volatile int* abort_flag = &bar.abort_flag;

  if (warp == 0) {
    if (lane == 0) {
      int bs = 0;
      uint32_t b_phase = 1;
      bool ok = true;
      for (int i = n0; i < n1 && ok; ++i) {
        for (int s = 0; s < count; ++s) {
          ok = ptx::mbar_wait(ptx::smem_u32(&bar.empty[bs]), b_phase, abort_flag);
          if (!ok) break;
          const uint32_t full = ptx::smem_u32(&bar.full[bs]);
          ptx::mbar_expect_tx(full, atoms * kAtomB);
          for (int k = 0; k < atoms; ++k)
            ptx::tma_load_2d(b_at + (bs * atoms + k) * kAtomB, &tm_b, full, k * 64, ids.list[s] * p.N + i * kBN);
          if (++bs == kBStages) { bs = 0; b_phase ^= 1u; }
        }
      }
      if (!ok) timed_out(p, 4);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && count > 0) {
      ptx::wait_for_previous_kernel();
      ptx::mbar_expect_tx(ptx::smem_u32(&bar.t_full), 2 * atoms * kAtomA);
      for (int term = 0; term < 2; ++term)
        for (int k = 0; k < atoms; ++k)
          ptx::tma_load_2d(a_at + (term * atoms + k) * kAtomA, &tm_t, ptx::smem_u32(&bar.t_full), k * 64,
                           static_cast<int>(term * p.rows + row0));
      const uint32_t idesc = ptx::idesc_bf16_f32(kTileRows, kBN);
      const int steps = (p.rank + 15) / 16;
      int bs = 0, acc = 0;
      uint32_t b_phase = 0, acc_phase = 1;
      bool ok = ptx::mbar_wait(ptx::smem_u32(&bar.t_full), 0, abort_flag);
      const int units = (n1 - n0) * count;
      for (int u = 0; u < units && ok; ++u) {
        ok = ptx::mbar_wait(ptx::smem_u32(&bar.full[bs]), b_phase, abort_flag) &&
             ptx::mbar_wait(ptx::smem_u32(&bar.acc_empty[acc]), acc_phase, abort_flag);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        for (int term = 0; term < 2; ++term) {
          for (int k = 0; k < steps; ++k) {
            const uint64_t a = ptx::smem_desc_sw128(a_at + (term * atoms + (k >> 2)) * kAtomA) + 2 * (k & 3);
            const uint64_t b = ptx::smem_desc_sw128(b_at + (bs * atoms + (k >> 2)) * kAtomB) + 2 * (k & 3);
            ptx::tc_mma_bf16(tmem + acc * kBN, a, b, idesc, term > 0 || k > 0);
          }
        }
        ptx::tc_commit(ptx::smem_u32(&bar.empty[bs]));
        ptx::tc_commit(ptx::smem_u32(&bar.acc_full[acc]));
        if (++bs == kBStages) { bs = 0; b_phase ^= 1u; }
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok) timed_out(p, 5);
    }
    __syncwarp();
  } else {
    ptx::wait_for_previous_kernel();
    const int quarter = warp & 3, r = quarter * 32 + lane, slot = ids.slot[r];
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    int ys = 0, acc = 0;
    uint32_t y_phase = 0, acc_phase = 0;
    bool ok = true;
    const bool idle = count == 0 && p.y_in == p.y_out;     // nothing to add and nothing to copy: what was asked for lands
    for (int i = 0; idle && i < ahead; ++i) ptx::mbar_wait(ptx::smem_u32(&bar.y_full[i]), 0, abort_flag);
    for (int i = n0; i < n1 && !idle; ++i) {
      ok = __all_sync(kFull, ptx::mbar_wait(ptx::smem_u32(&bar.y_full[ys]), y_phase, abort_flag));
      unsigned char* row = ybase + ys * kYBytes + r * 128;
      for (int s = 0; s < count && ok; ++s) {
        ok = __all_sync(kFull, ptx::mbar_wait(ptx::smem_u32(&bar.acc_full[acc]), acc_phase, abort_flag));
        const bool mine = slot == s;
        if (ok && __any_sync(kFull, mine)) {
          ptx::tc_fence_after_sync();
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t v[32];
            ptx::tmem_ld_32x32(lanes + acc * kBN + half * 32, v);
            ptx::tmem_ld_wait();
            if (mine) {
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                uint4* at = reinterpret_cast<uint4*>(row + (((half * 4 + c) ^ (r & 7)) << 4));
                uint4 y = *at;
                y.x = pair(low(y.x) + __uint_as_float(v[8 * c]), high(y.x) + __uint_as_float(v[8 * c + 1]));
                y.y = pair(low(y.y) + __uint_as_float(v[8 * c + 2]), high(y.y) + __uint_as_float(v[8 * c + 3]));
                y.z = pair(low(y.z) + __uint_as_float(v[8 * c + 4]), high(y.z) + __uint_as_float(v[8 * c + 5]));
                y.w = pair(low(y.w) + __uint_as_float(v[8 * c + 6]), high(y.w) + __uint_as_float(v[8 * c + 7]));
                *at = y;
              }
            }
          }
          ptx::tc_fence_before_sync();
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&bar.acc_empty[acc]));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok && lane == 0) timed_out(p, 6);
      ptx::fence_proxy_async_smem();
      if (epilogue_meets(!ok)) break;                    // one verdict for the four warps
      if (warp == 2 && lane == 0) {
        ptx::tma_store_2d(&tm_out, y_at + ys * kYBytes, i * kBN, static_cast<int>(row0));
        ptx::bulk_commit_group();
        if (i > n0 && i - 1 + ahead < n1) {                // the tile before this has left: a later one takes its place
          const int free = ys == 0 ? kYStages - 1 : ys - 1;
          const uint32_t y_full = ptx::smem_u32(&bar.y_full[free]);
          ptx::bulk_wait_group_read_but_one();
          ptx::mbar_expect_tx(y_full, kYBytes);
          ptx::tma_load_2d(y_at + free * kYBytes, &tm_in, y_full, (i - 1 + ahead) * kBN, static_cast<int>(row0));
        }
      }
      if (++ys == kYStages) { ys = 0; y_phase ^= 1u; }
    }
    if (warp == 2 && lane == 0) ptx::bulk_wait_group_read_all();
    __syncwarp();
  }
  finish(&bar, warp);
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

int shrink_smem(int stages) { return 1024 + stages * kStageBytes; }
int expand_smem(int rank) {
  const int atoms = (rank + 63) / 64;
  return 1024 + 2 * atoms * kAtomA + kYStages * kYBytes + kBStages * atoms * kAtomB;
}

// Parts of K: as many as two CTAs per SM take, at most a portable cluster.
int splits_of(const moe_ctx* ctx, long long rows, int K) {
  const long long tiles = (rows + kTileRows - 1) / kTileRows;
  const int blocks = (K + kBK - 1) / kBK;
  long long s = 2LL * ctx->num_sms / tiles;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s > blocks) s = blocks;
  return s < 1 ? 1 : static_cast<int>(s);
}

}  // namespace

namespace moe {

size_t adapter_tile_scratch_bytes(long long rows, int rank) { return static_cast<size_t>(rows) * rank * 4; }

moe_status launch_adapter_tiles(moe_ctx* ctx, AdapterParams p, cudaStream_t stream) {
  const int rank16 = (p.rank + 15) / 16 * 16;
  CUtensorMap tm_x, tm_a, tm_t, tm_b, tm_in, tm_out;
  if (!encode(ctx, &tm_x, p.x, p.rows, p.K, kTileRows) ||
      !encode(ctx, &tm_a, p.a, static_cast<uint64_t>(p.adapters) * p.rank, p.K, rank16) ||
      !encode(ctx, &tm_t, p.t, 2 * static_cast<uint64_t>(p.rows), p.rank, kTileRows) ||
      !encode(ctx, &tm_b, p.b, static_cast<uint64_t>(p.adapters) * p.N, p.rank, kBN) ||
      !encode(ctx, &tm_in, p.y_in, p.rows, p.N, kTileRows) || !encode(ctx, &tm_out, p.y_out, p.rows, p.N, kTileRows))
    return MOE_ERR_CUDA;
  p.splits = splits_of(ctx, p.rows, p.K);
  const long long tiles = (p.rows + kTileRows - 1) / kTileRows;
  const int stages = 3;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * p.splits));
  cfg.dynamicSmemBytes = shrink_smem(stages);
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(p.splits);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  if (cudaLaunchKernelEx(&cfg, adapter_shrink_tiles, tm_x, tm_a, p, stages, rank16) != cudaSuccess) return MOE_ERR_CUDA;
  const int n_tiles = (p.N - 1) / kBN + 1;
  long long groups = 2LL * ctx->num_sms / tiles;
  if (groups > n_tiles) groups = n_tiles;
  if (groups < 1) groups = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * groups));
  cfg.dynamicSmemBytes = expand_smem(p.rank);
  attr = cudaLaunchAttribute{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  ctx->last_launches += 2;
  return cudaLaunchKernelEx(&cfg, adapter_expand_tiles, tm_t, tm_b, tm_in, tm_out, p, static_cast<int>(groups)) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

cudaError_t prepare_adapter_tiles(moe_ctx* ctx) {
  (void)ctx;
  const cudaError_t e = cudaFuncSetAttribute(adapter_shrink_tiles, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             shrink_smem(kMaxStages));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(adapter_expand_tiles, cudaFuncAttributeMaxDynamicSharedMemorySize, expand_smem(128));
}

}  // namespace moe
