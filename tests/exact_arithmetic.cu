// Device arithmetic that the library's choices and codes rest on bit for bit, against the general operations.  Compiled and
// run by test_gpu_exact_arithmetic.py.  Every function returns how many results differ (or -1 for a failed launch).
#include "../paper_2607_23264_b200/csrc/blk_quant.cuh"
#include "../paper_2607_23264_b200/csrc/route_scored.cuh"

namespace {

__device__ uint32_t mix(uint32_t x) {          // a bijection of 32 bits, for varied operands
  x ^= x >> 16; x *= 0x7feb352du; x ^= x >> 15; x *= 0x846ca68bu; x ^= x >> 16;
  return x;
}
__device__ bool same(float a, float b) { return __float_as_uint(a) == __float_as_uint(b); }

// every mantissa of d in [1, 2), at exponent `e`
__global__ void reciprocals(int e, unsigned long long* differ) {
  const uint32_t m = blockIdx.x * blockDim.x + threadIdx.x;
  const float d = __uint_as_float((static_cast<uint32_t>(127 + e) << 23) | m);
  if (!same(moe::reciprocal_from_one(d), __frcp_rn(d))) atomicAdd(differ, 1ull);
}
// x from -80 to 106 in steps of 2^-17 and a little between them
__global__ void sigmoids(unsigned long long* differ) {
  const uint32_t i = blockIdx.x * blockDim.x + threadIdx.x;
  const float x = -moe::kNearSigmoid + (static_cast<float>(i) + static_cast<float>(mix(i) >> 8) * 0x1p-24f) * 0x1p-17f;
  if (!same(moe::route_sigmoid_near(fmaxf(x, -moe::kNearSigmoid)), moe::route_sigmoid(fmaxf(x, -moe::kNearSigmoid))))
    atomicAdd(differ, 1ull);
}
// quotients from 2^-12 (a quarter of the smallest code) to 448, for scales of every exponent the fast division takes; the
// operands are two hashes of a number of 32 bits whose top four are `part16`
__global__ void quotients(uint32_t part16, unsigned long long* differ) {
  const uint32_t i = blockIdx.x * blockDim.x + threadIdx.x, a = mix(i ^ (part16 << 28)), b = mix(a + 0x9e3779b9u);
  const float scale = __uint_as_float(((a % 190u + 37u) << 23) | (b & 0x7FFFFFu));                 // 2^-90 .. 2^99
  if (blk::general_scale(scale)) { atomicAdd(differ, 1ull); return; }
  const float part = __uint_as_float(((127u - (b >> 27) % 20u) << 23) | (mix(b) & 0x7FFFFFu));     // 2^-19 .. 2
  const float v = (a >> 31 ? -1.f : 1.f) * fminf(224.f * part, 448.f) * scale;
  const blk::FastDivider fast{scale, __frcp_rn(scale)};
  if (!same(fast(v), __fdiv_rn(v, scale))) atomicAdd(differ, 1ull);
}
// codes of the values next to where an E4M3 code ends: a midpoint of neighbouring codes times the scale, and four values on
// either side of it
__global__ void codes_at_boundaries(uint32_t seed, unsigned long long* differ) {
  const uint32_t i = blockIdx.x * blockDim.x + threadIdx.x, a = mix(i ^ seed);
  const float scale = __uint_as_float(((a % 190u + 37u) << 23) | (mix(a) & 0x7FFFFFu));
  const blk::FastDivider fast{scale, __frcp_rn(scale)};
  const blk::GeneralDivider general{scale};
  for (int c = 0; c < 126; ++c) {                            // between code c and c + 1
    const float lo = c < 8 ? c * 0x1p-9f : ldexpf(8 + (c & 7), (c >> 3) - 10);
    const float hi = c + 1 < 8 ? (c + 1) * 0x1p-9f : ldexpf(8 + ((c + 1) & 7), ((c + 1) >> 3) - 10);
    const uint32_t at = __float_as_uint(0.5f * (lo + hi) * scale);
    for (int n = -4; n <= 4; n += 3) {                       // (groups of four values)
      float v[4];
      for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(at + n + j - 1) * ((j & 1) ? -1.f : 1.f);
      if (blk::pack4(v, fast) != blk::pack4(v, general)) atomicAdd(differ, 1ull);
    }
  }
}

template <typename Launch>
long long count(Launch launch) {
  unsigned long long *d = nullptr, h = 0;
  if (cudaMalloc(&d, 8) != cudaSuccess) return -1;
  bool ok = cudaMemset(d, 0, 8) == cudaSuccess;
  if (ok) launch(d);
  ok = ok && cudaGetLastError() == cudaSuccess && cudaMemcpy(&h, d, 8, cudaMemcpyDeviceToHost) == cudaSuccess;
  cudaFree(d);
  return ok ? static_cast<long long>(h) : -1;
}

}  // namespace

extern "C" {
long long exact_reciprocals(int e) {
  return count([&](unsigned long long* d) { reciprocals<<<(1 << 23) / 256, 256>>>(e, d); });
}
long long exact_sigmoids() {
  return count([&](unsigned long long* d) { sigmoids<<<186 * (1 << 17) / 256, 256>>>(d); });
}
long long exact_quotients(uint32_t part16) {
  return count([&](unsigned long long* d) { quotients<<<1 << 20, 256>>>(part16, d); });
}
long long exact_codes(uint32_t seed) {
  return count([&](unsigned long long* d) { codes_at_boundaries<<<1 << 12, 256>>>(seed, d); });
}
}
