// Low-rank adapters of many requests added to a projection's output: y[r] += scale_i b_i (a_i x[r]), i the row's adapter.
//
// shrink : t = x a^T, a CTA per 16 rows and a part of K.  The adapters of its rows are taken one after the other, each read once
//          for all of its rows here; the other rows enter the product as zeros.  m16n8k16 products, operands straight from
//          global memory: a lane's 16 bytes of a row are eight neighbouring k, and as x and a are permuted along k alike, no
//          shuffle is needed.
// expand : y += scale t b^T, a CTA per 16 rows and 256 columns, a column per thread: fp32 dot products over the rank.
#include "adapters.cuh"

namespace {

using moe::AdapterParams;

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kRows = 16;                 // rows of a CTA
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxSplits = 16;

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// kTiles: tiles of eight ranks held in registers (rank <= 8 * kTiles).
template <int kTiles>
__global__ void __launch_bounds__(kThreads)
adapter_shrink(const AdapterParams p) {
  __shared__ int s_id[kRows];
  __shared__ float s_t[kWarps][kRows][8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  const long long row0 = static_cast<long long>(blockIdx.x) * kRows;
  const int split = blockIdx.y;
  if (threadIdx.x < kRows) s_id[threadIdx.x] = moe::adapter_of_row(p, p.offsets, p.adapter_of, row0 + threadIdx.x, split == 0);
  __syncthreads();
  const int my_id = s_id[lane & 15];
  unsigned left = __ballot_sync(kFull, my_id >= 0) & 0xFFFFu;
  // steps of 32 along K, dealt to the splits and then to the warps
  const int steps = (p.K + 31) / 32;
  const int s0 = static_cast<int>(static_cast<long long>(steps) * split / p.splits);
  const int s1 = static_cast<int>(static_cast<long long>(steps) * (split + 1) / p.splits);
  const int tiles = p.rank / 8;

  while (left) {
    const int first = __ffs(left) - 1, id = s_id[first];
    const unsigned mine = __ballot_sync(kFull, my_id == id) & 0xFFFFu;
    left &= ~mine;
    const bool lo = mine >> g & 1, hi = mine >> (g + 8) & 1;
    const __nv_bfloat16* xr = p.x + (row0 + g) * p.K + c * 8;
    const __nv_bfloat16* ar = p.a + (static_cast<size_t>(id) * p.rank + g) * p.K + c * 8;
    float acc[kTiles][4];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
    for (int s = s0 + warp; s < s1; s += kWarps) {
      const int k = s * 32;
      const bool in = k + c * 8 < p.K;
      uint4 xa = make_uint4(0u, 0u, 0u, 0u), xb = xa;
      if (in && lo) xa = __ldg(reinterpret_cast<const uint4*>(xr + k));
      if (in && hi) xb = __ldg(reinterpret_cast<const uint4*>(xr + static_cast<size_t>(8) * p.K + k));
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        if (j < tiles) {
          uint4 w = make_uint4(0u, 0u, 0u, 0u);
          if (in) w = __ldg(reinterpret_cast<const uint4*>(ar + static_cast<size_t>(8 * j) * p.K + k));
          mma_bf16(acc[j], xa.x, xb.x, xa.y, xb.y, w.x, w.y);
          mma_bf16(acc[j], xa.z, xb.z, xa.w, xb.w, w.z, w.w);
        }
      }
    }
    // the warps' sums in order, a tile of ranks at a time
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      if (j < tiles) {
        __syncthreads();
        s_t[warp][g][2 * c] = acc[j][0];
        s_t[warp][g][2 * c + 1] = acc[j][1];
        s_t[warp][g + 8][2 * c] = acc[j][2];
        s_t[warp][g + 8][2 * c + 1] = acc[j][3];
        __syncthreads();
        const int r = threadIdx.x >> 3, n = threadIdx.x & 7;
        if (threadIdx.x < kRows * 8 && (mine >> r & 1)) {
          float sum = 0.f;
          for (int w = 0; w < kWarps; ++w) sum += s_t[w][r][n];
          p.t[(static_cast<size_t>(split) * p.rows + row0 + r) * p.rank + 8 * j + n] = sum;
        }
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads)
adapter_expand(const AdapterParams p) {
  __shared__ int s_id[kRows];
  __shared__ float s_t[kRows][128];
  const int tid = threadIdx.x;
  const long long row0 = static_cast<long long>(blockIdx.x) * kRows;
  const int n = blockIdx.y * kThreads + tid;
  if (tid < kRows) s_id[tid] = moe::adapter_of_row(p, p.offsets, p.adapter_of, row0 + tid, false);
  __syncthreads();
  for (int i = tid; i < kRows * p.rank; i += kThreads) {
    const int r = i / p.rank, j = i - r * p.rank;
    const int id = s_id[r];
    float sum = 0.f;
    if (id >= 0) {
      for (int s = 0; s < p.splits; ++s) sum += p.t[(static_cast<size_t>(s) * p.rows + row0 + r) * p.rank + j];
      if (p.scale != nullptr) sum *= __ldg(p.scale + id);
    }
    s_t[r][j] = sum;
  }
  __syncthreads();
  if (n >= p.N) return;
  for (int r = 0; r < kRows && row0 + r < p.rows; ++r) {
    const size_t at = (row0 + r) * p.N + n;
    const int id = s_id[r];
    if (id < 0) {
      p.y_out[at] = p.y_in[at];
      continue;
    }
    const __nv_bfloat16* b = p.b + (static_cast<size_t>(id) * p.N + n) * p.rank;
    float sum = 0.f;
    for (int j = 0; j < p.rank; j += 8) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(b + j));
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum = fmaf(s_t[r][j + 2 * i], __uint_as_float(w[i] << 16), sum);
        sum = fmaf(s_t[r][j + 2 * i + 1], __uint_as_float(w[i] & 0xFFFF0000u), sum);
      }
    }
    p.y_out[at] = __float2bfloat16_rn(__bfloat162float(p.y_in[at]) + sum);
  }
}

// Parts of K: as many CTAs as fill the SMs about twice, each with at least four steps for a warp.
int splits_of(const moe_ctx* ctx, long long rows, int K) {
  const long long blocks = (rows + kRows - 1) / kRows;
  long long s = 2LL * ctx->num_sms / (blocks > 0 ? blocks : 1);
  const int most = (K + 32 * kWarps * 4 - 1) / (32 * kWarps * 4);
  if (s > most) s = most;
  if (s > kMaxSplits) s = kMaxSplits;
  return s < 1 ? 1 : static_cast<int>(s);
}

}  // namespace

namespace moe {

size_t adapter_scratch_bytes(const moe_ctx* ctx, long long rows, int K, int rank) {
  return static_cast<size_t>(splits_of(ctx, rows, K)) * static_cast<size_t>(rows) * rank * 4;
}

moe_status launch_add_adapters(moe_ctx* ctx, const moe_adapter_args& a, cudaStream_t stream) {
  AdapterParams p{};
  p.x = static_cast<const __nv_bfloat16*>(a.x);
  p.a = static_cast<const __nv_bfloat16*>(a.a);
  p.b = static_cast<const __nv_bfloat16*>(a.b);
  p.scale = a.scale;
  p.offsets = a.offsets;
  p.adapter_of = a.adapter_of;
  p.y_in = static_cast<const __nv_bfloat16*>(a.y_in);
  p.y_out = static_cast<__nv_bfloat16*>(a.y_out);
  p.t = static_cast<float*>(a.scratch);
  p.status = ctx->d_status;
  p.rows = a.rows;
  p.N = a.N;
  p.K = a.K;
  p.rank = a.rank;
  p.adapters = a.adapters;
  p.segments = a.segments;
  if (a.segments > 0 && a.rows >= 128 && a.rows / a.segments >= 16) return launch_adapter_tiles(ctx, p, stream);
  p.splits = splits_of(ctx, a.rows, a.K);
  const unsigned blocks = static_cast<unsigned>((a.rows + kRows - 1) / kRows);
  const unsigned chunks = static_cast<unsigned>((a.N - 1) / kThreads + 1);
  if (chunks > 65535u) return MOE_ERR_UNSUPPORTED_SHAPE;
  auto kernel = a.rank <= 16 ? adapter_shrink<2> : a.rank <= 32 ? adapter_shrink<4> : a.rank <= 64 ? adapter_shrink<8>
                                                                                               : adapter_shrink<16>;
  kernel<<<dim3(blocks, p.splits), kThreads, 0, stream>>>(p);
  if (cudaGetLastError() != cudaSuccess) return MOE_ERR_CUDA;
  adapter_expand<<<dim3(blocks, chunks), kThreads, 0, stream>>>(p);
  ctx->last_launches += 2;
  return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // namespace moe
