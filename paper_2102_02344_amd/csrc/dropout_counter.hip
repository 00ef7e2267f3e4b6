// Dropout whose mask is a function of the element's place (fusion rules table row "Dropout"; section "Our Proposal: HFTA", paragraph on
// per-model hyper-parameters: each model has its own rate and seed).
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel Random Numbers: As Easy as 1, 2, 3; SC 2011): ten rounds of two 32 x 32 -> 64 bit
// products turn a counter of four words and a key of two into four words.  Element i of model b takes word i % 4 of the
// block of counter (i / 4 low, i / 4 high, site, step) under the key seed[b], and is kept where that word, as a fraction of 2^32, is at
// least p[b].  The backward call forms the same words again: nothing is stored, and a model's mask does not depend on the models beside it.
//
// Bound by memory: 20 products for four elements stay below what a piece's 16 bytes in and out take (8 x 2097152 elements bf16: 14.2 us, 4.7 TB/s).
#include "pieces.h"

namespace hfta {
namespace {

struct DcArgs {
  const void* X;
  void* Y;
  const float* p;
  const uint64_t* seed;
  const uint32_t* step;
  int64_t count;
  uint32_t site;
};

__device__ __forceinline__ void dc_block(uint32_t (&w)[4], int64_t block, uint32_t site, uint32_t step, uint32_t k0, uint32_t k1) {
  w[0] = (uint32_t)block;
  w[1] = (uint32_t)((uint64_t)block >> 32);
  w[2] = site;
  w[3] = step;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t m = (uint64_t)0xD2511F53u * w[0], n = (uint64_t)0xCD9E8D57u * w[2];
    const uint32_t x = (uint32_t)(n >> 32) ^ w[1] ^ k0, z = (uint32_t)(m >> 32) ^ w[3] ^ k1;
    w[0] = x;
    w[1] = (uint32_t)n;
    w[2] = z;
    w[3] = (uint32_t)m;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

template <typename T> __global__ __launch_bounds__(256) void dc_kernel(DcArgs a) {
  typedef Piece16<T> P;
  const int b = blockIdx.y;
  const T* x = reinterpret_cast<const T*>(a.X) + b * a.count;
  T* y = reinterpret_cast<T*>(a.Y) + b * a.count;
  float p = a.p[b];
  p = p < 0.f ? 0.f : p > 1.f ? 1.f : p;                         // (a NaN stays one)
  const float f = 1.f / (1.f - p);
  // word >= p 2^32 in whole numbers; 2^32 itself, which keeps nothing, has no 32-bit form
  const uint32_t least = p < 1.f ? (uint32_t)__builtin_ceil((double)p * 4294967296.0) : 0xffffffffu;
  const bool none = p >= 1.f;
  const uint64_t seed = a.seed[b];
  const uint32_t step = a.step ? *a.step : 0u;
  const uint32_t k0 = __builtin_amdgcn_readfirstlane((uint32_t)seed), k1 = __builtin_amdgcn_readfirstlane((uint32_t)(seed >> 32));
  const int64_t stride = (int64_t)gridDim.x * 256 * P::N;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * P::N; i < a.count; i += stride) {
    const int n = (int)min((int64_t)P::N, a.count - i);
    float v[P::N];
    P::load(v, x + i, n);
#pragma unroll
    for (int q = 0; q < P::N / 4; ++q) {
      uint32_t w[4];
      dc_block(w, (i >> 2) + q, a.site, step, k0, k1);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = p != p ? p : w[e] >= least && !none ? f * v[4 * q + e] : 0.f;
    }
    P::store(y + i, v, n);
  }
}

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" int hfta_dropout_counter(int B, int64_t count, int dtype, const void* X, const float* p, const uint64_t* seed,
                                    const uint32_t* step, uint32_t site, void* Y, void* stream) {
  if (B <= 0 || count <= 0 || !valid_dtype(dtype) || !X || !p || !seed || !Y) return HFTA_EINVAL;
  if (count > ((int64_t)1 << 60) / B) return HFTA_EINVAL;
  if (B > 65535) return HFTA_EUNSUPPORTED;
  const DcArgs a{X, Y, p, seed, step, count, site};
  const int64_t per = 256 * (dtype == HFTA_BF16 ? 8 : 4), blocks = (count + per - 1) / per;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20), (unsigned)B);
  if (dtype == HFTA_BF16) hipLaunchKernelGGL(dc_kernel<bf16_raw>, grid, dim3(256), 0, as_stream(stream), a);
  else hipLaunchKernelGGL(dc_kernel<float>, grid, dim3(256), 0, as_stream(stream), a);
  return launch_status();
}
