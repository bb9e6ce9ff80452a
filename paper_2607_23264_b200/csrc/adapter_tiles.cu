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
constexpr int kMaxSplits = 16;

struct alignas(16) TileIds {
  int id[kTileRows];                      // adapter of each row, -1 without one
  int slot[kTileRows];                    // its place in `list`
  int list[kTileRows];                    // the tile's adapters in order of their first row
  int place[kTileRows];
  int warp_count[4];
  int32_t offsets[kCachedOffsets];
};
struct Barriers {
  uint64_t full[kMaxStages], empty[kMaxStages], y_full[kYStages], y_empty[kYStages], acc_full[2], acc_empty[2];
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

__global__ void __launch_bounds__(kThreads)
adapter_shrink_tiles(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_a, const AdapterParams p,
                     int stages, int rank16) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ TileIds ids;
  __shared__ Barriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile = blockIdx.x / p.splits, split = blockIdx.x - tile * p.splits;
  const long long row0 = static_cast<long long>(tile) * kTileRows;
  const uint32_t ring = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  ptx::launch_dependents();
  if (threadIdx.x == 0) {
    ptx::prefetch_tensormap(&tm_x);
    ptx::prefetch_tensormap(&tm_a);
    for (int i = 0; i < stages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.empty[i]), 1);
    }
    ptx::mbar_init(ptx::smem_u32(&bar.acc_full[0]), 1);
    ptx::mbar_init(ptx::smem_u32(&bar.acc_empty[0]), 4);
    bar.abort_flag = 0;
    ptx::fence_barrier_init();
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
  const int blocks = (p.K + kBK - 1) / kBK;
  const int kb0 = static_cast<int>(static_cast<long long>(blocks) * split / p.splits);
  const int kb1 = static_cast<int>(static_cast<long long>(blocks) * (split + 1) / p.splits);
  const int per_pass = kCols / rank16;                     // adapters

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 1;
      bool ok = true;
      for (int s0 = 0; s0 < count && ok; s0 += per_pass) {
        const int n = min(per_pass, count - s0);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!ptx::mbar_wait(ptx::smem_u32(&bar.empty[stage]), phase, abort_flag)) {
            timed_out(p, 1);
            ok = false;
            break;
          }
          const uint32_t full = ptx::smem_u32(&bar.full[stage]), at = ring + stage * kStageBytes;
          ptx::mbar_expect_tx(full, kXBytes + n * rank16 * 128);
          ptx::tma_load_2d(at, &tm_x, full, kb * kBK, static_cast<int>(row0));
          for (int i = 0; i < n; ++i)
            ptx::tma_load_2d(at + kXBytes + i * rank16 * 128, &tm_a, full, kb * kBK, ids.list[s0 + i] * p.rank);
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0, pass_phase = 1;
      bool ok = true;
      for (int s0 = 0; s0 < count && ok; s0 += per_pass) {
        const int n = min(per_pass, count - s0);
        const uint32_t idesc = ptx::idesc_bf16_f32(kTileRows, n * rank16);
        ok = ptx::mbar_wait(ptx::smem_u32(&bar.acc_empty[0]), pass_phase, abort_flag);
        pass_phase ^= 1u;
        ptx::tc_fence_after_sync();
        for (int kb = kb0; kb < kb1 && ok; ++kb) {
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
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, r = quarter * 32 + lane, slot = ids.slot[r];
    float* dst = p.t + (static_cast<size_t>(split) * p.rows + row0 + r) * p.rank;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    uint32_t phase = 0;
    for (int s0 = 0; s0 < count; s0 += per_pass) {
      const int n = min(per_pass, count - s0);
      if (!__all_sync(kFull, ptx::mbar_wait(ptx::smem_u32(&bar.acc_full[0]), phase, abort_flag))) {
        if (lane == 0) timed_out(p, 3);
        break;
      }
      phase ^= 1u;
      ptx::tc_fence_after_sync();
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
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&bar.acc_empty[0]));
    }
  }
  finish(&bar, warp);
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
adapter_expand_tiles(const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_in,
                     const __grid_constant__ CUtensorMap tm_out, const AdapterParams p, int groups) {
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
  if (threadIdx.x == 0) {
    ptx::prefetch_tensormap(&tm_b);
    ptx::prefetch_tensormap(&tm_in);
    ptx::prefetch_tensormap(&tm_out);
    for (int i = 0; i < kBStages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.empty[i]), 1);
    }
    for (int i = 0; i < kYStages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.y_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.y_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&bar.acc_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&bar.acc_empty[i]), 4);
    }
    bar.abort_flag = 0;
    ptx::fence_barrier_init();
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
  const int tiles = (p.N - 1) / kBN + 1;
  int n0 = static_cast<int>(static_cast<long long>(tiles) * group / groups);
  const int n1 = static_cast<int>(static_cast<long long>(tiles) * (group + 1) / groups);
  if (count == 0 && p.y_in == p.y_out) n0 = n1;            // nothing to add and nothing to copy

  if (warp == 0) {
    if (lane == 0) {
      int ys = 0, bs = 0;
      uint32_t y_phase = 1, b_phase = 1;
      bool ok = true;
      for (int i = n0; i < n1 && ok; ++i) {
        ok = ptx::mbar_wait(ptx::smem_u32(&bar.y_empty[ys]), y_phase, abort_flag);
        if (!ok) break;
        const uint32_t y_full = ptx::smem_u32(&bar.y_full[ys]);
        ptx::mbar_expect_tx(y_full, kYBytes);
        ptx::tma_load_2d(y_at + ys * kYBytes, &tm_in, y_full, i * kBN, static_cast<int>(row0));
        if (++ys == kYStages) { ys = 0; y_phase ^= 1u; }
        for (int s = 0; s < count && ok; ++s) {
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
  } else {
    // t, summed over the parts of K and scaled, as the A operand; eight ranks a step
    ptx::wait_for_previous_kernel();
    const int chunks = (p.rank + 15) / 16 * 2;             // 16-byte pieces of a row: whole steps of the product
    const int work = count > 0 && n0 < n1 ? kTileRows * chunks : 0;
    for (int i = threadIdx.x - 32; i < work; i += kThreads - 32) {
      const int r = i / chunks, j = i - r * chunks, id = ids.id[r];
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (id >= 0 && 8 * j < p.rank) {
        const float* src = p.t + static_cast<size_t>(row0 + r) * p.rank + 8 * j;
        const size_t pitch = static_cast<size_t>(p.rows) * p.rank;
        for (int s = 0; s < p.splits; ++s) {
          const float4 a = __ldcg(reinterpret_cast<const float4*>(src + s * pitch));
          const float4 b = __ldcg(reinterpret_cast<const float4*>(src + s * pitch) + 1);
          v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
          v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        }
        if (p.scale != nullptr) {
          const float f = __ldg(p.scale + id);
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] *= f;
        }
      }
      uint4 hi, lo;
      two_terms(v, hi, lo);
      unsigned char* at = base + (j >> 3) * kAtomA + r * 128 + (((j & 7) ^ (r & 7)) << 4);
      *reinterpret_cast<uint4*>(at) = hi;
      *reinterpret_cast<uint4*>(at + atoms * kAtomA) = lo;
    }
    ptx::fence_proxy_async_smem();
    asm volatile("bar.sync 1, %0;" ::"r"(kThreads - 32) : "memory");

    if (warp == 1) {
      if (lane == 0) {
        const uint32_t idesc = ptx::idesc_bf16_f32(kTileRows, kBN);
        const int steps = (p.rank + 15) / 16;
        int bs = 0, acc = 0;
        uint32_t b_phase = 0, acc_phase = 1;
        bool ok = true;
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
      const int quarter = warp & 3, r = quarter * 32 + lane, slot = ids.slot[r];
      const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
      int ys = 0, acc = 0;
      uint32_t y_phase = 0, acc_phase = 0;
      bool ok = true;
      for (int i = n0; i < n1; ++i) {
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
          ptx::bulk_wait_group_read_but_one();
          if (i > n0) ptx::mbar_arrive(ptx::smem_u32(&bar.y_empty[ys == 0 ? kYStages - 1 : ys - 1]));
        }
        if (++ys == kYStages) { ys = 0; y_phase ^= 1u; }
      }
      if (warp == 2 && lane == 0) ptx::bulk_wait_group_read_all();
      __syncwarp();
    }
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

}  // namespace

namespace moe {

int adapter_tile_splits(const moe_ctx* ctx, long long rows, int K, int) {
  const long long tiles = (rows + kTileRows - 1) / kTileRows;
  const int blocks = (K + kBK - 1) / kBK;
  long long s = tiles > 0 ? 2LL * ctx->num_sms / tiles : 1;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s > blocks) s = blocks;
  return s < 1 ? 1 : static_cast<int>(s);
}

moe_status launch_adapter_tiles(moe_ctx* ctx, AdapterParams p, cudaStream_t stream) {
  const int rank16 = (p.rank + 15) / 16 * 16;
  CUtensorMap tm_x, tm_a, tm_b, tm_in, tm_out;
  if (!encode(ctx, &tm_x, p.x, p.rows, p.K, kTileRows) ||
      !encode(ctx, &tm_a, p.a, static_cast<uint64_t>(p.adapters) * p.rank, p.K, rank16) ||
      !encode(ctx, &tm_b, p.b, static_cast<uint64_t>(p.adapters) * p.N, p.rank, kBN) ||
      !encode(ctx, &tm_in, p.y_in, p.rows, p.N, kTileRows) || !encode(ctx, &tm_out, p.y_out, p.rows, p.N, kTileRows))
    return MOE_ERR_CUDA;
  p.splits = adapter_tile_splits(ctx, p.rows, p.K, p.rank);
  const long long tiles = (p.rows + kTileRows - 1) / kTileRows;
  const int stages = 3;
  adapter_shrink_tiles<<<static_cast<unsigned>(tiles * p.splits), kThreads, shrink_smem(stages), stream>>>(tm_x, tm_a, p, stages,
                                                                                                  rank16);
  if (cudaGetLastError() != cudaSuccess) return MOE_ERR_CUDA;
  const int n_tiles = (p.N - 1) / kBN + 1;
  long long groups = 2LL * ctx->num_sms / tiles;
  if (groups > n_tiles) groups = n_tiles;
  if (groups < 1) groups = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * groups));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = expand_smem(p.rank);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  ctx->last_launches += 2;
  return cudaLaunchKernelEx(&cfg, adapter_expand_tiles, tm_b, tm_in, tm_out, p, static_cast<int>(groups)) == cudaSuccess
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
