// Grouped product of E4M3 rows and weights with fp32 scales per block of 128, and the two expert GEMMs on it:
//     y[r,n] = sum_b sa[b][r] sb[n/128][b] * P_b[r,n],     P_b[r,n] = sum_{k in block b} a[r,k] w[n,k]
// The scales are arbitrary fp32 numbers, which the tensor pipe cannot apply, so each block's P_b is an accumulator of its
// own in tensor memory (fp32), and epilogue warps add it, scaled, to the running sums in their registers while the
// tensor pipe computes the next block into the other half of tensor memory.  A tile is some rows of a group x 256
// accumulator columns: two weight boxes of 128 rows (Linear-1: 128 gate rows and the matching 128 up rows, so that a tile
// yields 128 columns of h, one whole block, which the epilogue quantises from the fp32 sums).
//
// Three kinds of tile, because the rows per group decide what bounds the work:
//   * few rows (at most 64): operands swapped.  The weight boxes are the M side of two MMAs, the rows, padded to 16, 32 or
//     64, their N side; an expert of few rows costs few multiply-adds, which under the power cap is what counts beside
//     the weights' bytes.  Each accumulator column has its own scale, read from shared memory.
//   * more rows (at most 128): the rows are the M side, an epilogue thread owns one row and a scale is one factor per
//     weight box (at 128 rows the swapped form's scale reads took as long as the sums).
//   * many rows per group: CTA pairs (clusters of two, cta_group::2) on tiles of 256 rows.  Each CTA stages its 128 rows
//     and one of the two weight boxes: 32 KB per block of K, 64 bytes per clock at the tensor rate, which is what an SM
//     takes in from L2, where a single CTA's 48 KB would need 96.  A single CTA keeps twice the weight bytes in flight,
//     which is what counts while the weights come from HBM (launch_product gives the measured rule).
// Shapes with too few tiles for the SMs split K over a cluster of up to eight CTAs, which add their running sums through
// distributed shared memory in rank order: no scratch memory, no atomics, the same bits every time.
//
// What bounds it and what it measured (E4M3 both, 2 x rows x N x K operations, events over back-to-back runs):
//   few rows: the weights' bytes.  64 groups of 2 rows, 2048 x 7168: 143 us, 6.56 TB/s; 17 rows, 4096 x 7168: 11.7 us,
//     of which about 5 are the launch and the cluster's sums.
//   128 rows a group, 64 groups, 2048 x 7168: 182 us, 5.6 TB/s, 1.3 PFLOP/s: the copies and the MMAs.  Without the drain's
//     multiply-adds, and without its loads from tensor memory too, it takes 177.
//   many rows: one group of 8192, 4096 x 7168: 224 us from rest.  Without the drain's loads from tensor memory 228, without
//     its multiply-adds 181, without both 162 (147 at twice the cuBLAS bf16 rate): 40 to 60 us are the multiply-adds: the
//     scale per block of 128 makes every accumulator leave tensor memory after four instructions and it is handed back when
//     seven eighths of it are added.  Under a long load the power cap bounds it (256 us sustained).  8 groups of 2048: 434 us,
//     2.2 PFLOP/s; 440, 361 and 333 in the same way.
//   16 groups of 256, 4096 x 4096: 88 us; without multiply-adds 80, without loads 84.
// Measured and not kept: prefetching the weights into L2 some blocks ahead (143 -> 180 us at 2 rows), 32 accumulator
// columns per load and packed pairs of multiply-adds (more registers, slower), sixteen epilogue warps.
//
// Roles (384 threads, 168 registers each at launch, moved to where they are needed): warp 0 = TMA producer, warps 1 and
// 3 = MMA issuers (even and odd blocks of K), warp 2 = scale loader (sa * sb per row and weight box, through a ring in
// shared memory), warps 4-11 = epilogue (four lane quarters x two halves; 128 running sums per thread at most).
// Every wait is bounded; a wait that gives up is reported through the status word and the CTA unwinds.
#include <cuda_bf16.h>

#include <type_traits>

#include "blk_quant.cuh"
#include "ffn_math.cuh"
#include "moe_internal.h"
#include "ptx_sm100.cuh"

namespace {

constexpr int kThreads = 384;
constexpr int kEpilogueThreads = 256;
constexpr int BW = 128;                  // rows of one weight box (M of an MMA)
constexpr int BK = 128;                  // K elements (= bytes) per block: one 128-byte swizzle row, one scale
constexpr int UMMA_K = 32;
constexpr int kWBoxBytes = BW * BK;
constexpr int kMaxStages = 6;
constexpr int kScaleSlots = 2;           // scale ring: slots of kScaleBatch blocks of K each
constexpr int kScaleBatch = 4;
constexpr int kScaleThreads = 32;
constexpr int kTmemCols = 512;           // two buffers x two weight boxes x 128 columns
constexpr int kTmemBuf = 256;
constexpr int kOutTokens = 8;            // swapped tiles: rows staged per step of the tile's end, per epilogue half
constexpr int kStoreBoxBytes = 32 * 64;  // other tiles: a warp's staging box, 32 rows x 64 bytes of output
constexpr int kStagingBytes = 2 * kOutTokens * 256 * 4;
static_assert(kStagingBytes == kEpilogueThreads / 32 * kStoreBoxBytes, "one staging area serves both");
constexpr int kSwapRows = 64;            // blocks of at most this many rows run with swapped operands
constexpr int kPartPitch = 260;          // floats per row of a K split's partial sums (conflict-free for both tile kinds)
constexpr int kMaxSmem = 227 * 1024;
constexpr int kKernelIdBlk = 10;         // in the detail word of a time-out: 10 * 65536 + role

struct BlkParams {
  const int32_t* offsets;   // [groups + 1] or null: one group of all rows
  int groups;
  int N;                    // output columns: F (Linear-1) or the product's N
  int n_tiles;              // column tiles: ceil(N / 128) gated, ceil(N / 256) otherwise
  int k_blocks;             // ceil(K / 128)
  int n_blocks;             // ceil(N / 128): pitch of the weight scales
  int rows;
  int stages;
  int split;                // CTAs per tile along K (the cluster size)
  const float* sa;          // [k_blocks][rows]
  const float* sb0;         // [groups][n_blocks][k_blocks]; gated: gate
  const float* sb1;         // gated: up
  __nv_bfloat16* y;         // [rows, N]: the product's one rounding.  In a layer it precedes the weighted sum of a token's rows,
                            // as in the library's other forms: combine then reads half the bytes of fp32 rows, and the
                            // rounding (1.7e-3 of the norm) joins that of the quantised h (3.5e-3) as independent error
  uint32_t* hq;             // gated: E4M3 [rows, N], four codes per word
  float* sh;                // gated: [N/128][rows]
  float* h_dbg;             // gated: optional fp32 [rows, N]
  int32_t* status;
};

// The rows of a, as boxes of each height a tile can have: one copy per block of K whatever the height (a copy costs the
// issuing warp about 100 clocks).
constexpr int kHeights = 5;
struct RowMaps {
  CUtensorMap of[kHeights];   // 16, 32, 64, 96, 128 rows
};
__host__ __device__ constexpr int blk_height(int i) { return i == 0 ? 16 : 32 * (i < 3 ? i : i < 4 ? 3 : 4); }
static_assert(blk_height(0) == 16 && blk_height(1) == 32 && blk_height(2) == 64 && blk_height(3) == 96 && blk_height(4) == 128, "");
__device__ __forceinline__ int blk_height_index(int rows) { return rows <= 16 ? 0 : rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 96 ? 3 : 4; }

struct BlkTail {
  uint64_t full[kMaxStages];
  uint64_t empty[kMaxStages];
  uint64_t acc_full[2];
  uint64_t acc_empty[2];
  uint64_t sc_full[kScaleSlots];
  uint64_t sc_empty[kScaleSlots];
  uint64_t out_sync[2];     // meeting points of an epilogue half's four warps (swapped tiles)
  uint64_t row_sync[4];     // meeting points of the two warps that share 32 rows
  uint32_t tmem_base;
  int abort_flag;
  float amax[2][2][BW];     // [tile parity][half][row]
};

// Per tile: kCtas CTAs x kMaxN rows of a.
template <int kCtas, int kMaxN>
struct BlkGeom {
  static constexpr int kWBoxes = kCtas == 2 ? 1 : 2;                        // weight boxes a CTA stages
  static constexpr int kRowsAt = kWBoxes * kWBoxBytes;                      // the rows' place in a stage
  static constexpr int kStageBytes = kRowsAt + kMaxN * BK;
};

struct BlkTile {
  int row0, rows;    // this CTA's rows of a: row0 .. row0 + rows - 1 (none: rows <= 0)
  int peer_rows;     // pairs: the other CTA's
  int n0;            // first output column
  int group;
  bool single;       // no other tile reads these weights
  bool swapped;
};

// The roles whose waits may give up; the flag holds the first that did, and the kernel's end reports it.
enum BlkRole { kRoleTma = 1, kRoleMma = 2, kRoleScale = 3, kRoleEpilogue = 4 };
__device__ __forceinline__ void blk_report(const BlkParams& p, int role) {
  atomicCAS(&p.status[0], 0, MOE_ERR_TIMEOUT);
  atomicCAS(&p.status[1], 0, kKernelIdBlk * 65536 + role);
}

// The group of tile t: the last one whose tiles start at or before it.  By a whole warp, 32 candidates at a time (two
// rounds for up to 1024 groups; a binary search by each lane cost 300 clocks per tile and role).
__device__ __forceinline__ int blk_group_of(int t, const int32_t* prefix, const BlkParams& p) {
  const int lane = threadIdx.x & 31;
  const int step = (p.groups + 31) >> 5;
  int i = lane * step;
  const uint32_t coarse = __ballot_sync(0xFFFFFFFFu, i < p.groups && prefix[min(i, p.groups)] * p.n_tiles <= t);
  const int base = (__popc(coarse) - 1) * step;
  i = base + lane;
  const uint32_t fine =
      __ballot_sync(0xFFFFFFFFu, lane < step && i < p.groups && prefix[min(i, p.groups)] * p.n_tiles <= t);
  return base + __popc(fine) - 1;
}

// Tile t of the list ordered by (group, chunk of column tiles, row block, column tile): the row blocks of a group and column
// tile run within one round of the CTAs and share the weight boxes in L2.  Pairs take chunks of sixteen (one group of 8192
// rows, 4096 x 7168: 221 us, 225 with eight, 231 with one, the row blocks next to each other).  Single CTAs take chunks of
// four, so that a group's short last block, which costs less, falls to other CTAs than its whole ones: with the row
// blocks next to each other and an even number of CTAs half of the CTAs get all the short ones (64 groups of 140 rows,
// 7168 x 2048: 330 us against 231, 243 with chunks of sixteen).
template <bool kGated, int kCtas, int kMaxN>
__device__ __forceinline__ BlkTile blk_decode(int t, int rank, const int32_t* prefix, const int32_t* offs,
                                              const BlkParams& p) {
  const int lo = blk_group_of(t, prefix, p);
  const int blocks = prefix[lo + 1] - prefix[lo];
  const int local = t - prefix[lo] * p.n_tiles;
  constexpr int kColChunk = kCtas == 2 ? 16 : 4;
  const int chunk = local / (blocks * kColChunk), in_chunk = local - chunk * blocks * kColChunk;
  const int width = min(kColChunk, p.n_tiles - chunk * kColChunk);
  const int mb = in_chunk / width, nb = chunk * kColChunk + in_chunk - mb * width;
  const int first = offs[2 * lo] + mb * kCtas * kMaxN;
  const int left = offs[2 * lo + 1] - first;                 // rows from this block on
  BlkTile tile;
  tile.row0 = first + rank * kMaxN;
  tile.rows = min(kMaxN, left - rank * kMaxN);
  tile.peer_rows = kCtas == 2 ? min(kMaxN, left - (rank ^ 1) * kMaxN) : 0;
  tile.n0 = nb * (kGated ? BW : 2 * BW);
  tile.group = lo;
  tile.single = blocks == 1;
  tile.swapped = kCtas == 1 && tile.rows <= kSwapRows;
  return tile;
}

// silu(g) * u to about 4 ulp: expf (2) and an approximate reciprocal (1).  h is quantised from here, and the error of the
// hardware tanh (2^-11) would move one code in a hundred.  32 groups of 128 rows, both GEMMs of 7168 / 2048: 281 us, 279
// with the exponential that grows by an ulp per unit of |g|, 289 with a division.
__device__ __forceinline__ float blk_silu_mul(float g, float u) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + expf(-g)));
  return g * r * u;
}

// One row of the output from its running sums: lane l holds columns n0 + 4 l .. + 3 of each weight box.
template <bool kGated>
__device__ __forceinline__ void blk_finish_row(const BlkParams& p, int row, int n0, int lane, const float4& a,
                                               const float4& b) {
  if constexpr (kGated) {
    const float g[4] = {a.x, a.y, a.z, a.w}, u[4] = {b.x, b.y, b.z, b.w};
    float h[4], amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = blk_silu_mul(g[i], u[i]);
      amax = fmaxf(amax, fabsf(h[i]));
    }
    amax = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(amax)));
    const float sc = blk::scale_of(amax);
    const size_t at = static_cast<size_t>(row) * p.N + n0 + 4 * lane;
    uint32_t w[1];
    blk::pack(h, sc, w);
    p.hq[at >> 2] = w[0];
    if (lane == 0) p.sh[static_cast<size_t>(n0 / BW) * p.rows + row] = sc;
    if (p.h_dbg != nullptr) *reinterpret_cast<float4*>(p.h_dbg + at) = make_float4(h[0], h[1], h[2], h[3]);
  } else {
    const int c0 = n0 + 4 * lane, c1 = c0 + BW;
    __nv_bfloat16* y = p.y + static_cast<size_t>(row) * p.N;
    if (c0 < p.N) *reinterpret_cast<uint2*>(y + c0) = make_uint2(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w));
    if (c1 < p.N) *reinterpret_cast<uint2*>(y + c1) = make_uint2(pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
  }
}

// One warp: row blocks (of `most` rows) before each group, and each group's first row and end.  Offsets are clamped:
// whatever they hold, no row outside [0, rows) is touched.
__device__ __forceinline__ void blk_prefixes(const BlkParams& p, int most, int32_t* prefix, int32_t* offs, int lane) {
  int32_t run = 0;
  for (int b0 = 0; b0 < p.groups; b0 += 32) {
    const int e = b0 + lane;
    int32_t v = 0;
    if (e < p.groups) {
      int32_t lo = p.offsets ? p.offsets[e] : 0, hi = p.offsets ? p.offsets[e + 1] : p.rows;
      lo = min(max(lo, 0), p.rows);
      hi = min(max(hi, lo), p.rows);
      offs[2 * e] = lo;
      offs[2 * e + 1] = hi;
      v = (hi - lo + most - 1) / most;
    }
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int32_t o = __shfl_up_sync(0xFFFFFFFFu, v, off);
      if (lane >= off) v += o;
    }
    if (e < p.groups) prefix[e + 1] = run + v;
    run += __shfl_sync(0xFFFFFFFFu, v, 31);
  }
}

// The scale loader's whole run: for kScaleBatch blocks of K at a time, row r of the tile gets sa * sb of each weight box in
// the next slot of the ring.  A slot's loads are in flight together and the ring lets the loader run ahead of the
// epilogue, across tiles too; the epilogue waits for scales once per slot.
template <bool kGated, int kCtas, int kMaxN>
__device__ __forceinline__ void blk_load_scales(const BlkParams& p, int rank, int first, int step, int total_tiles,
                                                int kb0, int kb1, int lane, const int32_t* prefix, const int32_t* offs,
                                                float* s_scale, BlkTail* st) {
  volatile int* abort_flag = &st->abort_flag;
  constexpr int kPer = (kMaxN + kScaleThreads - 1) / kScaleThreads;   // rows per thread
  int slot = 0;
  uint32_t slot_phase = 0;
  for (int t = first; t < total_tiles; t += step) {
    if (__any_sync(0xFFFFFFFFu, *abort_flag)) return;
    const BlkTile tile = blk_decode<kGated, kCtas, kMaxN>(t, rank, prefix, offs, p);
    const int nb = tile.n0 / BW;
    const size_t w_at = (static_cast<size_t>(tile.group) * p.n_blocks + nb) * p.k_blocks;
    const float* sb0 = p.sb0 + w_at;
    const float* sb1 = kGated ? p.sb1 + w_at : nb + 1 < p.n_blocks ? sb0 + p.k_blocks : nullptr;
    for (int kb = kb0; kb < kb1; kb += kScaleBatch) {
      float va[kScaleBatch][kPer], vb0[kScaleBatch], vb1[kScaleBatch];
#pragma unroll
      for (int u = 0; u < kScaleBatch; ++u) {
        const bool in = kb + u < kb1;
        vb0[u] = in ? __ldg(sb0 + kb + u) : 0.f;
        vb1[u] = in && sb1 ? __ldg(sb1 + kb + u) : 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int r = lane + i * kScaleThreads;
          va[u][i] = in && r < tile.rows ? __ldg(p.sa + static_cast<size_t>(kb + u) * p.rows + tile.row0 + r) : 0.f;
        }
      }
      ptx::mbar_wait_or_flag(ptx::smem_u32(&st->sc_empty[slot]), slot_phase ^ 1u, abort_flag, kRoleScale);
      float* f = s_scale + slot * kScaleBatch * 2 * kMaxN;
#pragma unroll
      for (int u = 0; u < kScaleBatch; ++u)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int r = lane + i * kScaleThreads;
          if (r < kMaxN) {
            f[u * 2 * kMaxN + r] = va[u][i] * vb0[u];
            f[u * 2 * kMaxN + kMaxN + r] = va[u][i] * vb1[u];
          }
        }
      ptx::mbar_arrive(ptx::smem_u32(&st->sc_full[slot]));
      if (++slot == kScaleSlots) { slot = 0; slot_phase ^= 1u; }
    }
  }
}

template <int kCols>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[kCols]) {
  if constexpr (kCols == 8) ptx::tmem_ld_32x8(taddr, r);
  else ptx::tmem_ld_32x16(taddr, r);
}

// acc[0 .. kCols) += P * f for kCols columns of tensor memory; f are the columns' scales in shared memory.
template <int kCols>
__device__ __forceinline__ void blk_add_cols(uint32_t taddr, const float* f, float* acc) {
  uint32_t v[kCols];
  tmem_ld_cols<kCols>(taddr, v);
  ptx::tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < kCols; i += 4) {
    const float4 s = *reinterpret_cast<const float4*>(f + i);
    acc[i] = fmaf(__uint_as_float(v[i]), s.x, acc[i]);
    acc[i + 1] = fmaf(__uint_as_float(v[i + 1]), s.y, acc[i + 1]);
    acc[i + 2] = fmaf(__uint_as_float(v[i + 2]), s.z, acc[i + 2]);
    acc[i + 3] = fmaf(__uint_as_float(v[i + 3]), s.w, acc[i + 3]);
  }
}

// 64 bytes of each of the warp's 32 rows (16 words per lane, its row) through the warp's box in shared memory, so that a
// store instruction covers 64 contiguous bytes of eight rows instead of 16 bytes of 32.  dst: the byte address of row 0 of
// the warp; rows and 16-byte pieces beyond `rows` and `pieces` are left out.  (A bulk copy from the box does it in fewer
// instructions, but the box cannot be filled again for some 600 clocks: 3800 clocks per tile against 1700.)
__device__ __forceinline__ void store_rows_64(unsigned char* box, const uint4 (&w)[4], unsigned char* dst, size_t pitch,
                                              int rows, int pieces, int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(box + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = w[i];
  __syncwarp();
  const int piece = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 8 * i + (lane >> 2);
    const uint4 q = *reinterpret_cast<const uint4*>(box + r * 64 + ((piece ^ ((r >> 1) & 3)) << 4));
    if (r < rows && piece < pieces) *reinterpret_cast<uint4*>(dst + r * pitch + 16 * piece) = q;
  }
  __syncwarp();
}

// What an epilogue warp carries from tile to tile.
struct EpilogueState {
  int buf = 0, slot = 0, parity = 0;
  uint32_t buf_phase = 0, slot_phase = 0, out_phase = 0, row_phase = 0;
};

// A tile with swapped operands: this thread's lane is a row of each weight box, its sums are kCols rows of a (one half of
// the tile's padded rows).  Either the tile's end, or, with K split, this CTA's sums to `part`.
template <bool kGated, int kMaxN, int kCols>
__device__ __forceinline__ void blk_swapped_tile(const BlkParams& p, const BlkTile& tile, int kb0, int kb1, uint32_t tmem_base,
                                                 const float* s_scale, float* s_out, float* part, BlkTail* st,
                                                 EpilogueState& es) {
  volatile int* abort_flag = &st->abort_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int quarter = warp & 3, half = (warp - 4) >> 2;
  float acc[2][kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) acc[0][i] = acc[1][i] = 0.f;
  const uint32_t t_lane = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(half * kCols);
  for (int kb = kb0; kb < kb1; kb += kScaleBatch) {
    ptx::mbar_wait_or_flag(ptx::smem_u32(&st->sc_full[es.slot]), es.slot_phase, abort_flag, kRoleEpilogue);
    const float* f = s_scale + es.slot * kScaleBatch * 2 * kMaxN + half * kCols;
    const int batch = min(kScaleBatch, kb1 - kb);
    for (int u = 0; u < batch; ++u, f += 2 * kMaxN) {
      ptx::mbar_wait_or_flag(ptx::smem_u32(&st->acc_full[es.buf]), es.buf_phase, abort_flag, kRoleEpilogue);
      ptx::tc_fence_after_sync();
      const uint32_t ta = t_lane + static_cast<uint32_t>(es.buf * kTmemBuf);
      constexpr int kChunk = kCols < 16 ? kCols : 16;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < kCols; c += kChunk) blk_add_cols<kChunk>(ta + b * BW + c, f + b * kMaxN + c, &acc[b][c]);
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive_if(ptx::smem_u32(&st->acc_empty[es.buf]), lane == 0);
      if (++es.buf == 2) { es.buf = 0; es.buf_phase ^= 1u; }
    }
    __syncwarp();
    ptx::mbar_arrive_if(ptx::smem_u32(&st->sc_empty[es.slot]), lane == 0);
    if (++es.slot == kScaleSlots) { es.slot = 0; es.slot_phase ^= 1u; }
  }
  if (part != nullptr) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
#pragma unroll
      for (int b = 0; b < 2; ++b) part[(half * kCols + i) * kPartPitch + b * BW + quarter * 32 + lane] = acc[b][i];
    return;
  }
  // the four warps of a half meet (a bounded wait: a plain barrier would hang on a warp that gave up)
  auto meet = [&]() {
    const uint32_t bar = ptx::smem_u32(&st->out_sync[half]);
    __syncwarp();
    ptx::mbar_arrive_if(bar, lane == 0);
    ptx::mbar_wait_or_flag(bar, es.out_phase, abort_flag, kRoleEpilogue);
    es.out_phase ^= 1u;
  };
  // kOutTokens rows at a time through shared memory: weight rows become neighbouring columns of an output row.  The half's
  // area of it also is its warps' boxes of a row tile (store_rows_64), and with one or two blocks of K nothing else holds a
  // warp back from the next tile's end while another still stores the last one's: so the warps meet before the first write
  // too, wherever tiles of both kinds can follow each other.
  float* mine = s_out + half * kOutTokens * 256;
  if constexpr (kMaxN > kSwapRows) meet();
#pragma unroll
  for (int c = 0; c < kCols; c += kOutTokens) {
    if (half * kCols + c >= tile.rows) break;            // (the same for the four warps of a half)
#pragma unroll
    for (int i = 0; i < kOutTokens; ++i)
#pragma unroll
      for (int b = 0; b < 2; ++b) mine[i * 256 + b * BW + quarter * 32 + lane] = acc[b][c + i];
    meet();
#pragma unroll
    for (int i = 0; i < kOutTokens / 4; ++i) {
      const int j = quarter * (kOutTokens / 4) + i, r = half * kCols + c + j;
      if (r < tile.rows) {
        const float4 a = *reinterpret_cast<const float4*>(mine + j * 256 + 4 * lane);
        const float4 b = *reinterpret_cast<const float4*>(mine + j * 256 + BW + 4 * lane);
        blk_finish_row<kGated>(p, tile.row0 + r, tile.n0, lane, a, b);
      }
    }
    meet();
  }
}

// A tile with the rows of a as the M side: this thread owns one row, its sums are columns 64 half .. + 63 of each weight box.
template <bool kGated, bool kPair>
__device__ __forceinline__ void blk_row_tile(const BlkParams& p, const BlkTile& tile, int kb0, int kb1, uint32_t tmem_base,
                                             uint32_t empty0, uint32_t empty1, const float* s_scale, unsigned char* s_store,
                                             float* part, BlkTail* st, EpilogueState& es) {
  volatile int* abort_flag = &st->abort_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int quarter = warp & 3, half = (warp - 4) >> 2;
  const int r_tile = quarter * 32 + lane;
  const uint32_t t_lane = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(half * 64);
  const int warp_rows = tile.rows - quarter * 32;         // the group's rows among this warp's 32 (may be more, or none)
  const bool live = warp_rows > 0;
  float acc[128];                                         // 0..63: the first box, 64..127: the second
#pragma unroll
  for (int i = 0; i < 128; ++i) acc[i] = 0.f;
  // the loop over the blocks of K, with the sums or (warps without rows) without: a branch inside it cost 5 %
  auto blocks = [&](auto with_sums) {
    for (int kb = kb0; kb < kb1; kb += kScaleBatch) {
      ptx::mbar_wait_or_flag(ptx::smem_u32(&st->sc_full[es.slot]), es.slot_phase, abort_flag, kRoleEpilogue);
      const float* f = s_scale + es.slot * kScaleBatch * 2 * BW + r_tile;
      const int batch = min(kScaleBatch, kb1 - kb);
      for (int u = 0; u < batch; ++u, f += 2 * BW) {
        const float s0 = f[0], s1 = f[BW];
        ptx::mbar_wait_or_flag(ptx::smem_u32(&st->acc_full[es.buf]), es.buf_phase, abort_flag, kRoleEpilogue);
        ptx::tc_fence_after_sync();
        const uint32_t empty = es.buf == 0 ? empty0 : empty1;
        auto hand_back = [&]() {
          ptx::tc_fence_before_sync();
          // in a pair the arrival crosses it, without a cluster-wide release (300 clocks more): the loads from tensor
          // memory have completed and there is nothing else to publish
          if constexpr (kPair) ptx::mbar_arrive_cluster_if(empty, lane == 0);
          else ptx::mbar_arrive_if(empty, lane == 0);
        };
        if constexpr (decltype(with_sums)::value) {
          const uint32_t ta = t_lane + static_cast<uint32_t>(es.buf * kTmemBuf);
          // the next 16 columns are on their way while the last 16 are added (32 at a time was 4 % slower: register moves)
          uint32_t v[2][16];
          ptx::tmem_ld_32x16(ta, v[0]);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            ptx::tmem_ld_wait();
            if (c < 7) ptx::tmem_ld_32x16(ta + ((c + 1) >> 2) * BW + ((c + 1) & 3) * 16, v[(c + 1) & 1]);
            else hand_back();                             // the warp's loads from this accumulator have completed
#pragma unroll
            for (int i = 0; i < 16; ++i)
              acc[16 * c + i] = fmaf(__uint_as_float(v[c & 1][i]), c < 4 ? s0 : s1, acc[16 * c + i]);
          }
        } else {
          hand_back();
        }
        if (++es.buf == 2) { es.buf = 0; es.buf_phase ^= 1u; }
      }
      __syncwarp();
      ptx::mbar_arrive_if(ptx::smem_u32(&st->sc_empty[es.slot]), lane == 0);
      if (++es.slot == kScaleSlots) { es.slot = 0; es.slot_phase ^= 1u; }
    }
  };
  if (live) blocks(std::true_type{});
  else blocks(std::false_type{});
  if (!kPair && part != nullptr) {
    float* dst = part + r_tile * kPartPitch + half * 64;
#pragma unroll
    for (int i = 0; i < 128; i += 4)
      *reinterpret_cast<float4*>(dst + (i >> 6) * BW + (i & 63)) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
    return;
  }
  const int row = tile.row0 + r_tile;
  unsigned char* box = s_store + (warp - 4) * kStoreBoxBytes;
  if constexpr (kGated) {
    float h[64], amax = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) {
      h[i] = blk_silu_mul(acc[i], acc[64 + i]);
      amax = fmaxf(amax, fabsf(h[i]));
    }
    // a block of h is 128 columns: the row's other 64 are the other half's
    st->amax[es.parity][half][r_tile] = amax;
    __syncwarp();
    const uint32_t bar = ptx::smem_u32(&st->row_sync[quarter]);
    ptx::mbar_arrive_if(bar, lane == 0);
    ptx::mbar_wait_or_flag(bar, es.row_phase, abort_flag, kRoleEpilogue);
    es.row_phase ^= 1u;
    amax = fmaxf(amax, st->amax[es.parity][half ^ 1][r_tile]);
    es.parity ^= 1;
    if (!live) return;
    const float sc = blk::scale_of(amax);
    const size_t at = static_cast<size_t>(row) * p.N + tile.n0 + half * 64;
    uint32_t codes[16];
    blk::pack(h, sc, codes);
    uint4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = make_uint4(codes[4 * i], codes[4 * i + 1], codes[4 * i + 2], codes[4 * i + 3]);
    store_rows_64(box, w, reinterpret_cast<unsigned char*>(p.hq) + at - static_cast<size_t>(lane) * p.N, p.N, warp_rows, 4, lane);
    if (lane < warp_rows) {
      if (half == 0) p.sh[static_cast<size_t>(tile.n0 / BW) * p.rows + row] = sc;
      if (p.h_dbg != nullptr) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          *reinterpret_cast<float4*>(p.h_dbg + at + 4 * i) = make_float4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
      }
    }
  } else if (live) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {                            // 32 columns at a time, two of each weight box
      const int col0 = tile.n0 + (c >> 1) * BW + half * 64 + (c & 1) * 32;
      if (col0 >= p.N) continue;
      uint4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* v = acc + 32 * c + 8 * i;
        w[i] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
      }
      store_rows_64(box, w, reinterpret_cast<unsigned char*>(p.y + static_cast<size_t>(row - lane) * p.N + col0),
                    static_cast<size_t>(p.N) * 2, warp_rows, (p.N - col0) / 8, lane);
    }
  }
}

template <bool kGated, int kCtas, int kMaxN>
__global__ void __launch_bounds__(kThreads, 1)
gemm_blk(const __grid_constant__ RowMaps tm_a, const __grid_constant__ CUtensorMap tm_b0,
         const __grid_constant__ CUtensorMap tm_b1, const BlkParams p) {
  using G = BlkGeom<kCtas, kMaxN>;
  constexpr bool kPair = kCtas == 2;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  unsigned char* base = smem_raw + pad;                      // 1024-byte aligned: required by the swizzle
  const uint32_t ring_u32 = raw + pad;
  unsigned char* s_staging = base + p.stages * G::kStageBytes;
  float* s_scale = reinterpret_cast<float*>(s_staging + kStagingBytes);        // [kScaleSlots][kScaleBatch][2][kMaxN]
  BlkTail* st = reinterpret_cast<BlkTail*>(s_scale + kScaleSlots * kScaleBatch * 2 * kMaxN);
  int32_t* prefix = reinterpret_cast<int32_t*>(st + 1);                        // [groups + 1] row blocks before a group
  int32_t* offs = prefix + p.groups + 1;                                       // [groups][2] first row, end

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool in_cluster = kPair || p.split > 1;
  const int cta = in_cluster ? static_cast<int>(ptx::cluster_ctarank()) : 0;
  const int rank = kPair ? cta : 0;                          // of a pair: 0 = leader, which issues the MMAs

  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) {
      ptx::mbar_init(ptx::smem_u32(&st->full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&st->empty[s]), 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(ptx::smem_u32(&st->acc_full[a]), 1);
      ptx::mbar_init(ptx::smem_u32(&st->acc_empty[a]), kCtas * kEpilogueThreads / 32);   // a pair: the warps of both CTAs
      ptx::mbar_init(ptx::smem_u32(&st->out_sync[a]), kEpilogueThreads / 64);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      ptx::mbar_init(ptx::smem_u32(&st->sc_full[s]), kScaleThreads);
      ptx::mbar_init(ptx::smem_u32(&st->sc_empty[s]), kEpilogueThreads / 32);
    }
    for (int q = 0; q < 4; ++q) ptx::mbar_init(ptx::smem_u32(&st->row_sync[q]), 2);
    st->abort_flag = 0;
    prefix[0] = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async_smem();
  }
  if (warp == 0) {
    blk_prefixes(p, kCtas * kMaxN, prefix, offs, lane);
    if (lane == 0) {
      for (int i = 0; i < kHeights && blk_height(i) <= kMaxN; ++i) ptx::prefetch_tensormap(&tm_a.of[i]);
      ptx::prefetch_tensormap(&tm_b0);
      if (kGated) ptx::prefetch_tensormap(&tm_b1);
    }
  }
  if (warp == 1) {
    if constexpr (kPair) {
      ptx::tmem_alloc_pair(ptx::smem_u32(&st->tmem_base), kTmemCols);
      ptx::tmem_relinquish_pair();
    } else {
      ptx::tmem_alloc(ptx::smem_u32(&st->tmem_base), kTmemCols);
      ptx::tmem_relinquish();
    }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (kPair) ptx::cluster_sync();   // both CTAs' barriers exist before anything signals across the pair
  ptx::tc_fence_after_sync();

  const uint32_t tmem_base = st->tmem_base;
  const int total_tiles = prefix[p.groups] * p.n_tiles;
  volatile int* abort_flag = &st->abort_flag;
  // this CTA's (pair's, cluster's) tiles and its part of K
  const int team = kPair ? 2 : p.split;
  const int first = blockIdx.x / team, step = gridDim.x / team;
  const int kb0 = kPair ? 0 : static_cast<int>(static_cast<long long>(cta) * p.k_blocks / p.split);
  const int kb1 = kPair ? p.k_blocks : static_cast<int>(static_cast<long long>(cta + 1) * p.k_blocks / p.split);
  auto decode = [&](int t) { return blk_decode<kGated, kCtas, kMaxN>(t, rank, prefix, offs, p); };

  // The TMA and MMA warps run their loops as a whole and one elected lane issues: with warp-uniform values the operands
  // already are in the registers such instructions read them from, which halves the cost against a single-lane branch.
  if (warp < 4) {
    ptx::setmaxnreg_dec<48>();
    if (warp == 0) {
      // ---------------------------------------------------------------- TMA producer
      int stage = 0;
      uint32_t phase = 1;
      const uint64_t pol_first = ptx::l2_policy_evict_first(), pol_last = ptx::l2_policy_evict_last();
      for (int t = first; t < total_tiles; t += step) {
        const BlkTile tile = decode(t);
        // The first box: gate rows, or the tile's first 128 columns; the second: up rows, or the next 128 columns where
        // there are any (a pair loads it anyway: what lies beyond N is computed and not stored, beyond the last group it
        // reads as zero).  In a pair the leader takes the first and the peer the second.
        const int w_row0 = tile.group * p.N + tile.n0, w_row1 = kGated ? w_row0 : w_row0 + BW;
        const bool second = kPair || kGated || tile.n0 + BW < p.N;
        const uint64_t pol_w = tile.single ? pol_first : pol_last;   // weights another tile reads again stay in L2
        const int my_rows = tile.rows > 0 ? blk_height(blk_height_index(tile.rows)) : 0;
        const int peer_rows = tile.peer_rows > 0 ? blk_height(blk_height_index(tile.peer_rows)) : 0;
        const uint32_t bytes = (second ? 2 : 1) * kWBoxBytes + (my_rows + peer_rows) * BK;   // of both CTAs
        const CUtensorMap* ma = &tm_a.of[blk_height_index(tile.rows)];
        for (int kb = kb0; kb < kb1; ++kb) {
          ptx::mbar_wait_or_flag(ptx::smem_u32(&st->empty[stage]), phase, abort_flag, kRoleTma);
          if (__any_sync(0xFFFFFFFFu, *abort_flag)) break;           // no copies into stages that are not free
          const uint32_t full = ptx::smem_u32(&st->full[stage]);
          const uint32_t s = ring_u32 + stage * G::kStageBytes;
          if constexpr (kPair) {
            const uint32_t full_leader = ptx::map_to_cta(full, 0);
            const CUtensorMap* mb = rank == 0 ? &tm_b0 : &tm_b1;
            if (ptx::elect_one()) {
              if (rank == 0) ptx::mbar_expect_tx(full, bytes);
              ptx::tma_load_2d_pair_hint(s, mb, full_leader, kb * BK, rank == 0 ? w_row0 : w_row1, pol_w);
              if (my_rows > 0) ptx::tma_load_2d_pair_hint(s + G::kRowsAt, ma, full_leader, kb * BK, tile.row0, pol_last);
            }
          } else if (ptx::elect_one()) {
            ptx::mbar_expect_tx(full, bytes);
            ptx::tma_load_2d_hint(s, &tm_b0, full, kb * BK, w_row0, pol_w);
            if (second) ptx::tma_load_2d_hint(s + kWBoxBytes, kGated ? &tm_b1 : &tm_b0, full, kb * BK, w_row1, pol_w);
            ptx::tma_load_2d_hint(s + G::kRowsAt, ma, full, kb * BK, tile.row0, pol_last);
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
        if (__any_sync(0xFFFFFFFFu, *abort_flag)) break;
      }
    } else if (warp != 2) {
      // ---------------------------------------------------------------- MMA issuers: warp 1 even blocks of K, warp 3 odd
      // A block's two waits, MMAs and commits are a chain of 450 to 700 clocks for the issuing warp, more while the
      // epilogue's sums share its scheduler; blocks accumulate apart, so two warps take them in turn.
      if (rank == 0) {
        const int odd = warp >> 1;
        int stage = 0, next = 0;                   // ring position, and which issuer takes it
        uint32_t phase = 0, buf_phase = 1;
        const uint32_t d = tmem_base + static_cast<uint32_t>(odd * kTmemBuf);
        for (int t = first; t < total_tiles; t += step) {
          if (__any_sync(0xFFFFFFFFu, *abort_flag)) break;
          const BlkTile tile = decode(t);
          const uint32_t idesc = tile.swapped ? ptx::idesc_e4m3_f32(BW, blk_height(blk_height_index(tile.rows)))
                                              : ptx::idesc_e4m3_f32(kCtas * BW, 2 * BW);
          for (int kb = kb0; kb < kb1; ++kb) {
            if (next == odd) {
              ptx::mbar_wait_or_flag(ptx::smem_u32(&st->acc_empty[odd]), buf_phase, abort_flag, kRoleMma);
              ptx::mbar_wait_or_flag(ptx::smem_u32(&st->full[stage]), phase, abort_flag, kRoleMma);
              buf_phase ^= 1u;
              ptx::tc_fence_after_sync();
              const uint32_t s = ring_u32 + stage * G::kStageBytes;
              const uint64_t w0 = ptx::smem_desc_sw128(s), w1 = ptx::smem_desc_sw128(s + kWBoxBytes);
              const uint64_t a = ptx::smem_desc_sw128(s + G::kRowsAt);
              if (ptx::elect_one()) {
                // +32 bytes along K inside the swizzle row per MMA; the two boxes lie one behind the other, so as the N
                // side they are one operand of 256 rows
                if constexpr (kPair) {
#pragma unroll
                  for (int k4 = 0; k4 < BK / UMMA_K; ++k4)
                    ptx::tc_mma_e4m3_pair(d, a + 2 * k4, w0 + 2 * k4, idesc, k4 != 0 ? 1u : 0u);
                  ptx::tc_commit_pair(ptx::smem_u32(&st->empty[stage]), 3);    // in both CTAs
                  ptx::tc_commit_pair(ptx::smem_u32(&st->acc_full[odd]), 3);
                } else {
                  if (tile.swapped) {
#pragma unroll
                    for (int k4 = 0; k4 < BK / UMMA_K; ++k4) {
                      ptx::tc_mma_e4m3(d, w0 + 2 * k4, a + 2 * k4, idesc, k4 != 0 ? 1u : 0u);
                      ptx::tc_mma_e4m3(d + BW, w1 + 2 * k4, a + 2 * k4, idesc, k4 != 0 ? 1u : 0u);
                    }
                  } else {
#pragma unroll
                    for (int k4 = 0; k4 < BK / UMMA_K; ++k4)
                      ptx::tc_mma_e4m3(d, a + 2 * k4, w0 + 2 * k4, idesc, k4 != 0 ? 1u : 0u);
                  }
                  ptx::tc_commit(ptx::smem_u32(&st->empty[stage]));
                  ptx::tc_commit(ptx::smem_u32(&st->acc_full[odd]));
                }
              }
              __syncwarp();
            }
            next ^= 1;
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
          }
        }
      }
    } else {
      blk_load_scales<kGated, kCtas, kMaxN>(p, rank, first, step, total_tiles, kb0, kb1, lane, prefix, offs, s_scale, st);
    }
    if (!kPair && p.split > 1) {
      __syncwarp();
      ptx::cluster_sync();
      ptx::cluster_sync();
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    ptx::setmaxnreg_inc<224>();
    EpilogueState es;
    uint32_t empty0 = ptx::smem_u32(&st->acc_empty[0]), empty1 = ptx::smem_u32(&st->acc_empty[1]);
    if constexpr (kPair) {
      empty0 = ptx::map_to_cta(empty0, 0);
      empty1 = ptx::map_to_cta(empty1, 0);
    }
    // With K split (one tile per cluster) the ring is idle once the last block's MMAs are done: it takes the partial sums.
    float* part = !kPair && p.split > 1 ? reinterpret_cast<float*>(base) : nullptr;
    float* s_out = reinterpret_cast<float*>(s_staging);
    BlkTile tile{};
    for (int t = first; t < total_tiles; t += step) {
      if (__any_sync(0xFFFFFFFFu, *abort_flag)) break;
      tile = decode(t);
      if (!tile.swapped) {
        if constexpr (kMaxN == BW)
          blk_row_tile<kGated, kPair>(p, tile, kb0, kb1, tmem_base, empty0, empty1, s_scale, s_staging, part, st, es);
      } else if constexpr (!kPair) {
        const int height = blk_height_index(tile.rows);
        if (height == 0) blk_swapped_tile<kGated, kMaxN, 8>(p, tile, kb0, kb1, tmem_base, s_scale, s_out, part, st, es);
        else if (height == 1) blk_swapped_tile<kGated, kMaxN, 16>(p, tile, kb0, kb1, tmem_base, s_scale, s_out, part, st, es);
        else if constexpr (kMaxN >= kSwapRows)
          blk_swapped_tile<kGated, kMaxN, 32>(p, tile, kb0, kb1, tmem_base, s_scale, s_out, part, st, es);
      }
      if (part != nullptr) break;
    }
    if (part != nullptr) {
      __syncwarp();
      ptx::cluster_sync();
      if (first < total_tiles) {
        // each CTA finishes every split-th row, its eight epilogue warps in turn; partial sums in rank order
        for (int r = cta + p.split * (warp - 4); r < tile.rows; r += p.split * (kEpilogueThreads / 32)) {
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
          for (int c = 0; c < p.split; ++c) {
            const uint32_t at = ptx::map_to_cta(ring_u32 + static_cast<uint32_t>(r * kPartPitch + 4 * lane) * 4, c);
            const float4 va = ptx::ld_cluster_f4(at), vb = ptx::ld_cluster_f4(at + BW * 4);
            a.x += va.x; a.y += va.y; a.z += va.z; a.w += va.w;
            b.x += vb.x; b.y += vb.y; b.z += vb.z; b.w += vb.w;
          }
          blk_finish_row<kGated>(p, tile.row0 + r, tile.n0, lane, a, b);
        }
      }
      __syncwarp();
      ptx::cluster_sync();
    }
  }

  __syncthreads();
  if (st->abort_flag) {
    if (tid == 0) blk_report(p, st->abort_flag);
    // a wait gave up: give copies still in flight time to land before the shared memory is released
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (kPair) ptx::cluster_sync();   // the peer's shared memory and barriers stay alive until both CTAs are done
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    if constexpr (kPair) ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
    else ptx::tmem_dealloc(tmem_base, kTmemCols);
  }
}

// Tensor map over a row-major [rows, cols] matrix of E4M3 bytes: boxes of box_rows x 128 bytes, 128-byte swizzle; what
// lies outside reads as zero.
CUresult encode_bytes(moe_ctx* ctx, CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows) {
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {cols};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(BK), box_rows};
  const cuuint32_t elem[2] = {1u, 1u};
  return ctx->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, elem,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

struct BlkProduct {       // one GEMM: operands and shape
  const void *a, *b0, *b1;
  int K;
};

bool encode_rows(moe_ctx* ctx, RowMaps* maps, const BlkProduct& g, int rows) {
  for (int i = 0; i < kHeights; ++i)
    if (encode_bytes(ctx, &maps->of[i], g.a, rows, g.K, blk_height(i)) != CUDA_SUCCESS) return false;
  return true;
}

// The most tiles the rows can make (exact for one group): ceil(r / b) <= (r - 1) / b + 1 for each of at most `some` groups
// with rows.  The kernel counts the real ones from the offsets.
long long most_tiles(const BlkParams& p, int block_rows) {
  const long long some = p.groups < p.rows ? p.groups : p.rows;
  return ((p.rows - some) / block_rows + some) * p.n_tiles;
}

// CTAs per tile along K: the most, up to eight, for which every tile's cluster is resident at once, and no more than give
// each CTA fewer blocks.  (A cluster lies within a GPC: sixteen clusters of eight do not fit, and a second wave costs more
// than the longer loops: 17 rows, 4096 x 7168 took 18 us with eight CTAs per tile and 12 with six, 96 CTAs.)
int k_split(const moe_ctx* ctx, long long tiles, int k_blocks) {
  int split = 8;
  while (split > 1 && (split > k_blocks || tiles > ctx->blk_clusters[split])) --split;
  while (split > 1 && (k_blocks + split - 2) / (split - 1) == (k_blocks + split - 1) / split) --split;
  return split;
}

template <bool kGated, int kCtas, int kMaxN>
moe_status launch_tiles(moe_ctx* ctx, const BlkProduct& g, BlkParams p, cudaStream_t stream) {
  using G = BlkGeom<kCtas, kMaxN>;
  const uint64_t w_rows = static_cast<uint64_t>(p.groups) * p.N;
  RowMaps tm_a;
  CUtensorMap tm_b0, tm_b1;
  if (!encode_rows(ctx, &tm_a, g, p.rows) || encode_bytes(ctx, &tm_b0, g.b0, w_rows, g.K, BW) != CUDA_SUCCESS ||
      encode_bytes(ctx, &tm_b1, kGated ? g.b1 : g.b0, w_rows, g.K, BW) != CUDA_SUCCESS)
    return MOE_ERR_CUDA;
  const size_t rest = 1024 + kStagingBytes + kScaleSlots * kScaleBatch * 2 * kMaxN * 4 + sizeof(BlkTail) +
                      (3 * static_cast<size_t>(p.groups) + 1) * 4 + 16;
  p.stages = static_cast<int>((kMaxSmem - rest) / G::kStageBytes);           // 3 to 6
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  const size_t smem = rest + static_cast<size_t>(p.stages) * G::kStageBytes;
  const long long tiles = most_tiles(p, kCtas * kMaxN);
  p.split = kCtas == 2 ? 1 : k_split(ctx, tiles, p.k_blocks);
  const int team = kCtas == 2 ? 2 : p.split;
  const long long room = kCtas == 2 ? ctx->max_pairs : ctx->num_sms / team;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(team * (tiles < room ? tiles : room)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = team;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = team > 1 ? 1 : 0;
  ctx->last_launches += 1;
  return cudaLaunchKernelEx(&cfg, gemm_blk<kGated, kCtas, kMaxN>, tm_a, tm_b0, tm_b1, p) == cudaSuccess ? MOE_OK
                                                                                                     : MOE_ERR_CUDA;
}

template <bool kGated>
moe_status launch_product(moe_ctx* ctx, const BlkProduct& g, const BlkParams& p, cudaStream_t stream) {
  // By the average rows per group, us, equal groups, CTA pairs / single CTAs:
  //     64 groups, 2048 x 7168:  128 rows 238/185   192 251/246   256 265/276   300 448/361   384 507/388   512 527/496
  //      8 groups, 4096 x 7168:  512 rows 127/132   600 177/161   700 181/184   800 216/209  1024 225/236  2048 434/461
  //     16 groups, 7168 x 2048:  512 rows 142/145  1024 260/272  2048 500/529
  // A pair's tile has 256 rows, and the last of a group is padded to them: from about four full tiles on, the pair's 2 to
  // 6 % outweigh that whatever the remainder (a layer of 64 experts with 128 rows each on average: 3.50 ms with pairs,
  // 2.59 ms without).
  const long long pair_rows = moe_knob_value(ctx, "blk_pair_rows", 900);   // (0: pairs for every product, for tests)
  // Single CTAs with boxes of at most 32 rows have room for five stages, those of 128 rows for four, which do more rows
  // with each read of the weights; us, 32 / 128: 64 groups, 2048 x 7168: 2 rows 144.7/149.8, 16 144.7/148.2, 32
  // 147.3/151.2, 40 164.6/154.3; 128 groups, 7168 x 2048: 2 rows 281/281, 16 287/286, 24 300/296, 32 314/303.  On average
  // 16, because groups above 32 rows are the rule when the average is 32.
  const long long few_rows = moe_knob_value(ctx, "blk_few_rows", 16);
  if (p.rows > pair_rows * p.groups) {
    // Where the pairs have one tile each at most, single CTAs with K split may be done sooner (their blocks of K take
    // about a fifth longer): 512 rows, 4096 x 7168.
    const long long pair_tiles = most_tiles(p, 256), tiles = most_tiles(p, 128);
    const int split = k_split(ctx, tiles, p.k_blocks);
    if (pair_rows == 0 || pair_tiles > ctx->max_pairs || tiles > ctx->num_sms ||
        6LL * ((p.k_blocks + split - 1) / split) >= 5LL * p.k_blocks)
      return launch_tiles<kGated, 2, 128>(ctx, g, p, stream);
    return launch_tiles<kGated, 1, 128>(ctx, g, p, stream);
  }
  if (p.rows > few_rows * p.groups) return launch_tiles<kGated, 1, 128>(ctx, g, p, stream);
  return launch_tiles<kGated, 1, 32>(ctx, g, p, stream);
}

}  // namespace

namespace moe {

cudaError_t prepare_gemm_blk(moe_ctx* ctx) {
  const void* kernels[] = {
      reinterpret_cast<const void*>(gemm_blk<true, 1, 32>),  reinterpret_cast<const void*>(gemm_blk<false, 1, 32>),
      reinterpret_cast<const void*>(gemm_blk<true, 1, 128>), reinterpret_cast<const void*>(gemm_blk<false, 1, 128>),
      reinterpret_cast<const void*>(gemm_blk<true, 2, 128>), reinterpret_cast<const void*>(gemm_blk<false, 2, 128>)};
  for (const void* k : kernels) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    if (e != cudaSuccess) return e;
  }
  for (int n = 1; n <= 8; ++n) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(n);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kMaxSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = n;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&ctx->blk_clusters[n], gemm_blk<false, 1, 128>, &cfg);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

moe_status launch_gemm_blk(moe_ctx* ctx, const moe_gemm_blk_args* a, cudaStream_t stream) {
  BlkParams p{};
  p.offsets = a->offsets;
  p.groups = a->groups;
  p.N = a->N;
  p.n_tiles = blocks_of(a->N, 2 * BW);
  p.k_blocks = blocks_of(a->K, BK);
  p.n_blocks = blocks_of(a->N, BW);
  p.rows = static_cast<int>(a->rows);
  p.sa = a->sa;
  p.sb0 = a->sb;
  p.y = static_cast<__nv_bfloat16*>(a->y);
  p.status = ctx->d_status;
  return launch_product<false>(ctx, BlkProduct{a->a, a->b, a->b, a->K}, p, stream);
}

moe_status launch_expert_ffn_blk(moe_ctx* ctx, const moe_blk_ffn_args* a, cudaStream_t stream) {
  const moe_shape& s = ctx->shape;
  BlkParams p{};
  p.offsets = a->offsets;
  p.groups = s.E;
  p.rows = static_cast<int>(static_cast<long long>(s.T) * s.k);
  p.status = ctx->d_status;
  BlkParams p1 = p;
  p1.N = s.F;
  p1.n_tiles = p1.n_blocks = s.F / BW;
  p1.k_blocks = s.H / BK;
  p1.sa = a->sx_perm;
  p1.sb0 = a->s_gate;
  p1.sb1 = a->s_up;
  p1.hq = static_cast<uint32_t*>(a->hq_ws);
  p1.sh = a->sh_ws;
  p1.h_dbg = a->h_fp32_debug;
  moe_status st = launch_product<true>(ctx, BlkProduct{a->xq_perm, a->wq_gate, a->wq_up, s.H}, p1, stream);
  if (st != MOE_OK) return st;
  moe_mark(ctx, 5, stream);
  BlkParams p2 = p;
  p2.N = s.H;
  p2.n_tiles = blocks_of(s.H, 2 * BW);
  p2.n_blocks = s.H / BW;
  p2.k_blocks = s.F / BK;
  p2.sa = a->sh_ws;
  p2.sb0 = a->s_down;
  p2.y = static_cast<__nv_bfloat16*>(a->y_perm);
  st = launch_product<false>(ctx, BlkProduct{a->hq_ws, a->wq_down, a->wq_down, s.F}, p2, stream);
  if (st != MOE_OK) return st;
  moe_mark(ctx, 6, stream);
  return MOE_OK;
}

}  // namespace moe
