// Linear attention with a decay for each key head, one token at a time (linear_attention.h has the form for whole sequences):
//
//   S' = lambda S + k v^T,   ctx = scale q S'       lambda = exp(log_decay)
//
// A state is d x d fp32 and is read and written whole for each token, which is all that bounds this: 8 d^2 bytes beside a few rows of
// d.  A workgroup takes one token and key head with all query heads of its group.  A row of the state lies across lanes, four columns
// each, and a lane's share of it (16 rows at d = 128) is in flight at once; the sums over rows pass through LDS.  8 x 96 tokens, 16 heads of 128 over 8,
// bf16: 168 us, 4.8 TB/s, the rate of a large copy; 2 x 3 tokens of 4 heads of 64: 8.7 us, of which the kernel 5.
//
// lambda goes in as its fp32 value and the rest: a rounded lambda alone would change the rate at which a state forgets by 2^-25 / |log_decay|, the
// same way in every step.
//
// Rows of a call that name the same slot are tokens of one sequence, in order: the workgroup of the first takes them all, the others
// find an earlier one and end.  (No two workgroups touch one state.)
#include "pieces.h"

#include <math.h>

namespace hfta {
namespace {

struct LsStr { int64_t b, r, h; };
struct LsArgs {
  const void *Q, *K, *V;
  const int32_t* slot;
  const float *ld, *S;
  float* S2;
  void* CTX;
  LsStr qs, ks, cs;
  int n, slots, Hq, Hkv, d;
  float scale;
};

// D: columns that a row of the state is padded to; W: columns of a lane
template <typename T, int D, int W> __global__ __launch_bounds__(256) void ls_kernel(LsArgs a) {
  constexpr int LANES = D / W, GROUPS = 256 / LANES, RPT = (D + GROUPS - 1) / GROUPS;      // rows of a thread
  constexpr int HB = 4;                                          // query heads at a time
  typedef float vec __attribute__((ext_vector_type(W)));
  __shared__ float sk[D], sv[D], sq[HB][D], part[HB][GROUPS][D];
  __shared__ int later;
  const int t = threadIdx.x, cl = t % LANES, rg = t / LANES, c0 = cl * W, d = a.d;
  const int hk = blockIdx.x % a.Hkv, i = blockIdx.x / a.Hkv, b = blockIdx.y, G = a.Hq / a.Hkv;
  const int32_t* slot = a.slot ? a.slot + (int64_t)b * a.n : nullptr;
  const int s = slot ? slot[i] : i;
  if (s < 0 || s >= a.slots) return;
  const int64_t at = (((int64_t)b * a.slots + s) * a.Hkv + hk) * d * d;
  const float* src = a.S + at;
  float* dst = a.S2 + at;
  const float g = a.ld[(int64_t)b * a.Hkv + hk], lambda = expf(g > 0.f ? 0.f : g);
  const float rest = lambda >= 0.5f ? expm1f(g > 0.f ? 0.f : g) - (lambda - 1.f) : 0.f;       // (the difference is exact)
  const bool has = c0 < d;                                       // (W divides d, or is 1)
  vec st[RPT];
#pragma unroll
  for (int j = 0; j < RPT; ++j) {
    const int r = rg + j * GROUPS;
    if (has && r < d) st[j] = *reinterpret_cast<const vec*>(src + r * d + c0);
    else st[j] = vec{};
  }
  if (slot) {                                                    // an earlier row of this slot takes this one too
    int before = 0;
    for (int j = t; j < i; j += 256) before |= slot[j] == s;
    if (__syncthreads_or(before)) return;
  }
  for (int row = i; row < a.n;) {
    const T* k = reinterpret_cast<const T*>(a.K) + b * a.ks.b + row * a.ks.r + hk * a.ks.h;
    const T* v = reinterpret_cast<const T*>(a.V) + b * a.ks.b + row * a.ks.r + hk * a.ks.h;
    __syncthreads();
    if (t == 0) later = a.n;
    for (int c = t; c < D; c += 256) {
      sk[c] = c < d ? Elem<T>::load(k + c) : 0.f;
      sv[c] = c < d ? Elem<T>::load(v + c) : 0.f;
    }
    __syncthreads();
    if (slot) {
      int next = a.n;
      for (int j = row + 1 + t; j < a.n; j += 256)
        if (slot[j] == s) { next = j; break; }
      if (next < a.n) atomicMin(&later, next);
    }
    vec vv;
#pragma unroll
    for (int e = 0; e < W; ++e) vv[e] = sv[c0 + e];
#pragma unroll
    for (int j = 0; j < RPT; ++j) {
      const int r = rg + j * GROUPS;
      if (has && r < d) {
        st[j] = lambda * st[j] + (rest * st[j] + sk[r] * vv);
        *reinterpret_cast<vec*>(dst + r * d + c0) = st[j];
      }
    }
    for (int g0 = 0; g0 < G; g0 += HB) {
      const int heads = min(HB, G - g0);
      const T* q = reinterpret_cast<const T*>(a.Q) + b * a.qs.b + row * a.qs.r + (int64_t)(hk * G + g0) * a.qs.h;
      if (g0) __syncthreads();                                   // the sums of the heads before have been read
      for (int c = t; c < heads * D; c += 256) sq[c / D][c % D] = c % D < d ? Elem<T>::load(q + (int64_t)(c / D) * a.qs.h + c % D) : 0.f;
      __syncthreads();
      for (int h = 0; h < heads; ++h) {
        vec o{};
#pragma unroll
        for (int j = 0; j < RPT; ++j) {
          const int r = rg + j * GROUPS;
          if (r < d) o += sq[h][r] * st[j];
        }
#pragma unroll
        for (int e = 0; e < W; ++e) part[h][rg][c0 + e] = o[e];
      }
      __syncthreads();
      for (int c = t; c < heads * D; c += 256) {
        const int h = c / D, col = c % D;
        if (col >= d) continue;
        float o = 0.f;
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) o += part[h][j][col];
        Elem<T>::store(reinterpret_cast<T*>(a.CTX) + b * a.cs.b + row * a.cs.r + (int64_t)(hk * G + g0 + h) * a.cs.h + col, a.scale * o);
      }
    }
    row = slot ? later : a.n;                                    // (every thread has passed a barrier since `later` was formed)
  }
}

template <typename T> int ls_launch(const LsArgs& a, int B, bool four, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.n * a.Hkv), (unsigned)B), block(256);
#define LS_LAUNCH(D)                                                                            \
  if (four) hipLaunchKernelGGL((ls_kernel<T, D, 4>), grid, block, 0, st, a);                    \
  else hipLaunchKernelGGL((ls_kernel<T, D, 1>), grid, block, 0, st, a);
  if (a.d <= 32) { LS_LAUNCH(32) }
  else if (a.d <= 64) { LS_LAUNCH(64) }
  else { LS_LAUNCH(128) }
#undef LS_LAUNCH
  return launch_status();
}

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" int hfta_linear_attention_step(int B, int n, int slots, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3],
                                          const void* K, const void* V, const int64_t kvs[3], const int32_t* slot,
                                          const float* log_decay, float scale, const float* state, void* CTX, const int64_t cs[3],
                                          float* new_state, void* stream) {
  if (B <= 0 || n <= 0 || slots <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv || !valid_dtype(dtype) || !isfinite(scale) || !Q || !qs ||
      !K || !V || !kvs || !log_decay || !state || !CTX || !cs || !new_state || (!slot && n > slots))
    return HFTA_EINVAL;
  if (d > 128 || B > 65535 || (int64_t)n * Hkv > 0xffffff) return HFTA_EUNSUPPORTED;
  LsArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.slot = slot; a.ld = log_decay; a.S = state; a.S2 = new_state; a.CTX = CTX;
  a.qs = LsStr{qs[0], qs[1], qs[2]}; a.ks = LsStr{kvs[0], kvs[1], kvs[2]}; a.cs = LsStr{cs[0], cs[1], cs[2]};
  a.n = n; a.slots = slots; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.scale = scale;
  const bool four = d % 4 == 0 && ((reinterpret_cast<uintptr_t>(state) | reinterpret_cast<uintptr_t>(new_state)) & 15) == 0;
  if (dtype == HFTA_BF16) return ls_launch<bf16_raw>(a, B, four, as_stream(stream));
  return ls_launch<float>(a, B, four, as_stream(stream));
}
