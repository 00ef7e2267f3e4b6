// Linear attention with a decay for each key head over packed sequences:
//
//   S_t = lambda S_t-1 + k_t v_t^T,   ctx_t = scale q_t S_t            lambda = exp(log_decay), S in front of a sequence: state_in, or zeros
//
// Forward and backward are sums of one form, f(A, B, C)_t = sum_{s <= t} lambda^(t-s) (a_t . b_s) c_s, taken from the first row to the last or back:
//   ctx = scale f(q, k, v);   dq = scale f(dctx, v, k);   from the last row: dv = scale f(k, q, dctx), dk = scale f(v, dctx, q), over a group's heads
// A workgroup walks one sequence of one head with the state in LDS, a thread a column of it.
#include "packed_rows.h"

#include <math.h>

namespace hfta {
namespace {

struct LaStr { int64_t b, r, h; };
struct LaJob {
  const void *A, *B, *C;
  void* O;
  LaStr as, bs, cs, os;
  const float* S0;
  float* S1;
  int rev, flip;                   // flip: the state's rows and columns change places in memory
};
struct LaArgs {
  LaJob job[3];
  const int32_t* off;
  const float* ld;
  int R, nseq, Hq, Hkv, d;
  float scale;
};

template <typename T> __global__ __launch_bounds__(128) void la_walk_kernel(LaArgs a, int jobs) {
  __shared__ float S[128 * 129], sa[128], sb[128], sc[128];
  const int c = threadIdx.x, d = a.d, G = a.Hq / a.Hkv;
  const int j = blockIdx.z, b = blockIdx.y, hk = blockIdx.x % a.Hkv, s = blockIdx.x / a.Hkv;
  const LaJob& J = a.job[j];
  const int32_t* off = a.off + (int64_t)b * (a.nseq + 1);
  const int lo = min(max(off[s], 0), a.R), hi = min(max(off[s + 1], lo), a.R);
  const float g = a.ld[(int64_t)b * a.Hkv + hk], lambda = expf(g > 0.f ? 0.f : g);
  const int64_t at = (((int64_t)b * a.nseq + s) * a.Hkv + hk) * d * d;
  for (int i = c; i < d * d; i += 128) S[(i / d) * 129 + i % d] = J.S0 ? J.flip ? J.S0[at + (i % d) * d + i / d] : J.S0[at + i] : 0.f;
  __syncthreads();
  for (int n = 0; n < hi - lo; ++n) {
    const int r = J.rev ? hi - 1 - n : lo + n;
    const int heads_b = J.rev ? G : 1, heads_a = J.rev ? 1 : G;
    // forward, the state decays before a row is added; backward, S0 is the gradient of the state behind the last row
    if (c < d && (!J.rev || n > 0))
      for (int i = 0; i < d; ++i) S[i * 129 + c] *= lambda;
    for (int h = 0; h < heads_b; ++h) {
      __syncthreads();
      const int hb = J.rev ? hk * G + h : hk;
      if (c < d) {
        sb[c] = Elem<T>::load(reinterpret_cast<const T*>(J.B) + b * J.bs.b + r * J.bs.r + hb * J.bs.h + c) * (J.rev ? a.scale : 1.f);
        sc[c] = Elem<T>::load(reinterpret_cast<const T*>(J.C) + b * J.cs.b + r * J.cs.r + hb * J.cs.h + c);
      }
      __syncthreads();
      if (c < d)
        for (int i = 0; i < d; ++i) S[i * 129 + c] = fmaf(sb[i], sc[c], S[i * 129 + c]);
    }
    for (int h = 0; h < heads_a; ++h) {
      __syncthreads();
      const int ha = J.rev ? hk : hk * G + h;
      if (c < d) sa[c] = Elem<T>::load(reinterpret_cast<const T*>(J.A) + b * J.as.b + r * J.as.r + ha * J.as.h + c);
      __syncthreads();
      if (c < d && J.O) {
        float o = 0.f;
        for (int i = 0; i < d; ++i) o = fmaf(sa[i], S[i * 129 + c], o);
        Elem<T>::store(reinterpret_cast<T*>(J.O) + b * J.os.b + r * J.os.r + ha * J.os.h + c, J.rev ? o : a.scale * o);
      }
    }
  }
  __syncthreads();
  if (J.S1)
    for (int i = c; i < d * d; i += 128) {
      const float x = S[(i / d) * 129 + i % d] * (J.rev && hi > lo ? lambda : 1.f);
      J.S1[J.flip ? at + (i % d) * d + i / d : at + i] = x;
    }
}

LaStr la_str(const int64_t* s) { return LaStr{s[0], s[1], s[2]}; }

int la_check(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  if (B <= 0 || R <= 0 || nseq <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv || !valid_dtype(dtype) || R > 0x7fffffff - 4096) return HFTA_EINVAL;
  return d > 128 || nseq > PACKED_MAX || B > 65535 || (int64_t)nseq * Hkv > 0xffffff ? HFTA_EUNSUPPORTED : HFTA_OK;
}

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" {

size_t hfta_linear_attention_fwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) { return 0; }
size_t hfta_linear_attention_bwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) { return 0; }

int hfta_linear_attention_fwd(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3], const void* K,
                              const void* V, const int64_t kvs[3], const int32_t* seq_offsets, const float* log_decay, float scale,
                              const float* state_in, void* CTX, const int64_t cs[3], float* state_out, void* workspace, size_t ws_bytes,
                              void* stream) {
  const int rc = la_check(B, R, nseq, Hq, Hkv, d, dtype);
  if (rc == HFTA_EINVAL || !Q || !qs || !K || !V || !kvs || !seq_offsets || !log_decay || !(scale > 0.f) || !isfinite(1.f / scale) || !CTX || !cs)
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  LaArgs a{};
  a.off = seq_offsets; a.ld = log_decay; a.R = R; a.nseq = nseq; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.scale = scale;
  a.job[0] = LaJob{Q, K, V, CTX, la_str(qs), la_str(kvs), la_str(kvs), la_str(cs), state_in, state_out, 0, 0};
  const dim3 grid((unsigned)(nseq * Hkv), (unsigned)B, 1);
  if (dtype == HFTA_BF16) hipLaunchKernelGGL(la_walk_kernel<bf16_raw>, grid, dim3(128), 0, as_stream(stream), a, 1);
  else hipLaunchKernelGGL(la_walk_kernel<float>, grid, dim3(128), 0, as_stream(stream), a, 1);
  return launch_status();
}

int hfta_linear_attention_bwd(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3], const void* K,
                              const void* V, const int64_t kvs[3], const int32_t* seq_offsets, const float* log_decay, float scale,
                              const float* state_in, const void* dCTX, const int64_t cs[3], const float* dstate_out, void* dQ,
                              const int64_t dqs[3], void* dK, void* dV, const int64_t dkvs[3], float* dstate_in, void* workspace,
                              size_t ws_bytes, void* stream) {
  const int rc = la_check(B, R, nseq, Hq, Hkv, d, dtype);
  if (rc == HFTA_EINVAL || !Q || !qs || !K || !V || !kvs || !seq_offsets || !log_decay || !(scale > 0.f) || !isfinite(1.f / scale) || !dCTX || !cs ||
      !dQ || !dqs || !dK || !dV || !dkvs)
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  LaArgs a{};
  a.off = seq_offsets; a.ld = log_decay; a.R = R; a.nseq = nseq; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.scale = scale;
  a.job[0] = LaJob{dCTX, V, K, dQ, la_str(cs), la_str(kvs), la_str(kvs), la_str(dqs), state_in, nullptr, 0, 1};
  a.job[1] = LaJob{K, Q, dCTX, dV, la_str(kvs), la_str(qs), la_str(cs), la_str(dkvs), dstate_out, dstate_in, 1, 0};
  a.job[2] = LaJob{V, dCTX, Q, dK, la_str(kvs), la_str(cs), la_str(qs), la_str(dkvs), dstate_out, nullptr, 1, 1};
  const dim3 grid((unsigned)(nseq * Hkv), (unsigned)B, 3);
  if (dtype == HFTA_BF16) hipLaunchKernelGGL(la_walk_kernel<bf16_raw>, grid, dim3(128), 0, as_stream(stream), a, 3);
  else hipLaunchKernelGGL(la_walk_kernel<float>, grid, dim3(128), 0, as_stream(stream), a, 3);
  return launch_status();
}

}  // extern "C"
