// Log-probabilities of packed sequences, and the loss of preferred pairs with the gradient of its logits (appendix
// "Fused Loss": a model's loss is the mean over its own pairs, its hyper-parameters are entries of device arrays).
//
//   lp_r = z_r[y_r] - log sum_k exp z_r[k],   L_s = sum of lp_r over the rows of sequence s that have a label
//   t_p = beta ((L_2p - ref_2p) - (L_2p+1 - ref_2p+1)),  loss = mean_p (1 - eps) softplus(-t_p) + eps softplus(t_p)
//   dz_r[k] = c_s (1[k = y_r] - softmax(z_r)_k),  c_2p = -c_2p+1 = -beta ((1 - eps) sigma(-t_p) - eps sigma(t_p)) / pairs
//
// Bound by memory: the gradient's factor needs the whole sequence, so rows with a label are read twice and every row of
// a sequence is written once; rows without one are not read.  A workgroup takes a row, or a wavefront one where rows are
// narrow, with 16-byte pieces from its first aligned element on.  Sums over a sequence are taken in 64 bits: the loss is a difference of long sums.
//
// Measured, bf16: 8 x 2048 rows of 8192 classes: rows 26 to 32 us, pairs 5, gradient 57; 4 x 4096 rows of 32001: 139, 5
// and 282 (1.05 GB of logits).  Pieces of 16 bytes, four in flight a thread (eight: 25 -> 33 us).
#include "packed_rows.h"

namespace hfta {
namespace {

constexpr float PF_LOG2E = 1.4426950408889634f;

// A row of K values: `head` up to the first 16-byte boundary, nv whole pieces, `tail` past the last
template <typename T> struct PfRow {
  static constexpr int EPP = 16 / (int)sizeof(T);
  int head, nv, tail;
  __device__ __forceinline__ PfRow(const T* z, int K) {
    const int off = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
    head = off ? min(K, EPP - off) : 0;
    nv = (K - head) / EPP;
    tail = K - head - nv * EPP;
  }
};
__device__ __forceinline__ void pf_unpack(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void pf_unpack(const uint4& v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ uint4 pf_pack(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ uint4 pf_pack(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
// exp(x - top), top >= x.  The difference first: it is exact or rounded by its own size, where the rounding of top log2(e) would be a factor common
// to all terms of a row, as large as the logits are (1000 of them around 1000: log-probabilities off by 4e-5, this way 1e-6).
__device__ __forceinline__ float pf_exp(float x, float top) { return __builtin_amdgcn_exp2f((x - top) * PF_LOG2E); }

// which of its workgroup's rows NT threads take
template <int NT> __device__ __forceinline__ int pf_row_of() { return NT == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0; }

// rows [lo, hi) of sequence s
__device__ __forceinline__ void pf_rows(const int32_t* off, int s, int R, int& lo, int& hi) {
  lo = min(max(off[s], 0), R);
  hi = min(max(off[s + 1], 0), R);
}

// ------------------------------------------------------------------ rows: the label's log-probability, and what the gradient needs of a row:
// its largest value, and one over the sum of the exponentials of distances from it.  (Joined as log-sum-exp they would be rounded as one number: a
// probability formed from that is off by as much as the logits are large, and can pass 1.)
template <typename T, int NT>
__global__ __launch_bounds__(256) void pf_rows_kernel(const T* __restrict__ logits, const int32_t* __restrict__ labels,
                                                      const int32_t* __restrict__ off, int nseq, float* __restrict__ top,
                                                      float* __restrict__ inv, float* __restrict__ lp, int R, int K) {
  constexpr int EPP = PfRow<T>::EPP, NV = 4;
  __shared__ float sm[4], ss[4];
  const int r = blockIdx.x * (256 / NT) + pf_row_of<NT>(), b = blockIdx.y, t = threadIdx.x % NT;
  const int64_t row = (int64_t)b * R + r;
  off += (int64_t)b * (nseq + 1);
  if (r >= R || r < off[0] || r >= off[nseq]) return;
  const int y = labels[row];
  if (y < 0) {
    if (t == 0) lp[row] = 0.f;
    return;
  }
  const T* z = logits + row * K;
  const PfRow<T> g(z, K);
  const uint4* zv = reinterpret_cast<const uint4*>(z + g.head);
  float m = -INFINITY, s = 0.f;
  auto take = [&](float mt, auto&& each) {          // joins values with maximum mt
    const float mn = fmaxf(m, mt), mu = mn == -INFINITY ? 0.f : mn;
    s *= pf_exp(m, mu);
    m = mn;
    each(mu);
  };
  for (int v0 = t; v0 < g.nv; v0 += NT * NV) {
    float x[NV][EPP];
    float mt = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (v0 + NT * j < g.nv) pf_unpack(zv[v0 + NT * j], x[j]);
      else
#pragma unroll
        for (int e = 0; e < EPP; ++e) x[j][e] = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < EPP; ++e) mt = fmaxf(mt, x[j][e]);
    take(mt, [&](float mu) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (v0 + NT * j < g.nv)                     // (512 bf16 columns are one of a lane's four pieces: 44 -> 32 us for 131072 rows)
#pragma unroll
          for (int e = 0; e < EPP; ++e) s += pf_exp(x[j][e], mu);
    });
  }
  if (t < g.head + g.tail) {
    const float x = Elem<T>::load(z + (t < g.head ? t : K - g.tail + t - g.head));
    take(x, [&](float mu) { s += pf_exp(x, mu); });
  }
  float M = m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  if constexpr (NT > 64) {
    if ((t & 63) == 0) sm[t >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  }
  const float Mu = M == -INFINITY ? 0.f : M;
  s = wave_sum(s * pf_exp(m, Mu));
  if constexpr (NT > 64) {
    if ((t & 63) == 0) ss[t >> 6] = s;
    __syncthreads();
    s = (ss[0] + ss[1]) + (ss[2] + ss[3]);
  }
  if (t == 0) {
    if (top) {
      top[row] = M;
      inv[row] = 1.f / s;
    }
    lp[row] = (label_score(z, y, K) - M) - logf(s);  // the two large terms first
  }
}

// a workgroup's sum over rows [lo, hi), in 64 bits: each thread eight rows at once, so that a sequence of many rows is no chain of
// loads; sh: four words of LDS, one per wavefront
__device__ __forceinline__ double pf_sum(const float* lp, int lo, int hi, double* sh) {
  constexpr int NV = 8;
  const int t = threadIdx.x;
  double v = 0;
  for (int i = lo + t; i < hi; i += 256 * NV) {
    float x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j] = i + 256 * j < hi ? lp[i + 256 * j] : 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) v += (double)x[j];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((t & 63) == 0) sh[t >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__global__ __launch_bounds__(256) void pf_seq_kernel(const float* __restrict__ lp, const int32_t* __restrict__ off, int nseq,
                                                     float* __restrict__ logps, int R) {
  __shared__ double sh[4];
  const int b = blockIdx.y, s = blockIdx.x;
  int lo, hi;
  pf_rows(off + (int64_t)b * (nseq + 1), s, R, lo, hi);
  const double v = pf_sum(lp + (int64_t)b * R, lo, hi, sh);
  if (threadIdx.x == 0) logps[(int64_t)b * nseq + s] = (float)v;
}

// ------------------------------------------------------------------ pairs: a workgroup each
// w x: a weight of zero takes no part, however large x is (a rejected text that the model rules out)
__device__ __forceinline__ double pf_part(double w, double x) { return w == 0.0 ? 0.0 : w * x; }

__global__ __launch_bounds__(256) void pf_pair_kernel(const float* __restrict__ lp, const int32_t* __restrict__ off, int pairs, const float* __restrict__ ref,
                                                      const float* __restrict__ beta, const float* __restrict__ smoothing,
                                                      float* __restrict__ logps, float* __restrict__ term, float* __restrict__ coef,
                                                      int R) {
  __shared__ double sh[2][4];
  const int b = blockIdx.y, p = blockIdx.x, nseq = 2 * pairs;
  off += (int64_t)b * (nseq + 1);
  lp += (int64_t)b * R;
  int lo[2], hi[2];
  double v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    pf_rows(off, 2 * p + i, R, lo[i], hi[i]);
    v[i] = pf_sum(lp, lo[i], hi[i], sh[i]);
  }
  const int64_t at = (int64_t)b * nseq + 2 * p;
  const double be = beta[b], eps = smoothing ? smoothing[b] : 0.f;
  const double t = be * ((v[0] - (double)ref[at]) - (v[1] - (double)ref[at + 1]));
  const double e = exp(-fabs(t)), tail = log1p(e);                  // softplus(x) = max(x, 0) + log1p(exp(-|x|))
  const double up = (t >= 0 ? 1.0 : e) / (1.0 + e), down = (t >= 0 ? e : 1.0) / (1.0 + e);      // sigma(t), sigma(-t)
  const float c = (float)(-be * ((1.0 - eps) * down - eps * up) / pairs);
  if (threadIdx.x == 0) {
    logps[at] = (float)v[0];
    logps[at + 1] = (float)v[1];
    term[(int64_t)b * pairs + p] = (float)(pf_part(1.0 - eps, fmax(-t, 0.0) + tail) + pf_part(eps, fmax(t, 0.0) + tail));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
    for (int r = lo[i] + (int)threadIdx.x; r < hi[i]; r += 256)
      coef[(int64_t)b * R + r] = i ? -c : c;
}

// ------------------------------------------------------------------ gradient: a row per workgroup; the last one of a
// model adds its pairs' terms (in order)
template <typename T, int NT>
__global__ __launch_bounds__(256) void pf_grad_kernel(const T* logits, const int32_t* __restrict__ labels,
                                                      const int32_t* __restrict__ off, int pairs, const float* __restrict__ top,
                                                      const float* __restrict__ inv, const float* __restrict__ coef,
                                                      const float* __restrict__ term, float* __restrict__ loss, T* dlogits, int R, int K) {
  constexpr int EPP = PfRow<T>::EPP, NV = 4;
  __shared__ double sh[4];
  // the last rows first: what the pass before read last may still be in the last-level cache
  const int b = (int)(gridDim.y - 1 - blockIdx.y), nseq = 2 * pairs, t = threadIdx.x % NT;
  if (blockIdx.x == 0) {
    const int t = threadIdx.x;
    double v = 0;
    for (int i = t; i < pairs; i += 256) v += (double)term[(int64_t)b * pairs + i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((t & 63) == 0) sh[t >> 6] = v;
    __syncthreads();
    if (t == 0) loss[b] = (float)(((sh[0] + sh[1]) + (sh[2] + sh[3])) / pairs);
    return;
  }
  const int r = R - (int)((blockIdx.x - 1) * (256 / NT) + pf_row_of<NT>()) - 1;
  if (r < 0) return;
  const int64_t row = (int64_t)b * R + r;
  off += (int64_t)b * (nseq + 1);
  if (r < off[0] || r >= off[nseq]) return;
  const int y = labels[row];
  const T* z = logits + row * K;
  T* dz = dlogits + row * K;
  const PfRow<T> g(dz, K);
  uint4* dv = reinterpret_cast<uint4*>(dz + g.head);
  if (y < 0) {
    for (int v = t; v < g.nv; v += NT) dv[v] = make_uint4(0, 0, 0, 0);
    if (t < g.head + g.tail) Elem<T>::store(dz + (t < g.head ? t : K - g.tail + t - g.head), 0.f);
    return;
  }
  const float c = coef[row], M = top[row], is = inv[row];
  auto grad = [&](float x, int k) { return c * fmaf(-pf_exp(x, M), is, k == y ? 1.f : 0.f); };
  if (((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0) {
    const uint4* zv = reinterpret_cast<const uint4*>(z + g.head);
    for (int v0 = t; v0 < g.nv; v0 += NT * NV) {
      uint4 u[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (v0 + NT * j < g.nv) u[j] = zv[v0 + NT * j];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int v = v0 + NT * j;
        if (v >= g.nv) continue;
        float x[EPP];
        pf_unpack(u[j], x);
#pragma unroll
        for (int e = 0; e < EPP; ++e) x[e] = grad(x[e], g.head + v * EPP + e);
        dv[v] = pf_pack(x);
      }
    }
    if (t < g.head + g.tail) {
      const int k = t < g.head ? t : K - g.tail + t - g.head;
      Elem<T>::store(dz + k, grad(Elem<T>::load(z + k), k));
    }
  } else {                                           // logits and gradient lie differently against 16 bytes
    for (int k = t; k < K; k += NT) Elem<T>::store(dz + k, grad(Elem<T>::load(z + k), k));
  }
}

int pf_check(int B, int R, int K, int nseq, int dtype) {
  if (B <= 0 || R <= 0 || K <= 0 || nseq <= 0 || !valid_dtype(dtype)) return HFTA_EINVAL;
  return B > 65535 || R > 0xfffffe || nseq > PACKED_MAX ? HFTA_EUNSUPPORTED : HFTA_OK;      // (a launch has fewer than 2^32 threads)
}

// A wavefront takes a row of up to 4 KB at once, four pieces a lane.  A workgroup each and a wavefront each, log-probabilities and loss of
// bf16 rows (8 models, 16 pairs, 60 % of the rows with a label): 131072 of 512 classes 91 / 32 and 177 / 66 us, 32768 of 2048 29 / 19 and 60 / 49,
// 16384 of 8192 28 / 32 and 93 / 103; fp32 rows of 512 classes 89 / 34 and 193 / 97, of 2048 31 / 26 and 93 / 97.
bool pf_narrow(int K, size_t es) { return (size_t)K * es <= 4096; }

template <typename T>
void pf_rows_launch(int B, int R, int K, int nseq, const void* logits, const int32_t* labels, const int32_t* off, float* top,
                    float* inv, float* lp, hipStream_t st) {
  if (pf_narrow(K, sizeof(T)))
    hipLaunchKernelGGL((pf_rows_kernel<T, 64>), dim3((unsigned)(R + 3) / 4, (unsigned)B), dim3(256), 0, st, (const T*)logits, labels, off,
                       nseq, top, inv, lp, R, K);
  else
    hipLaunchKernelGGL((pf_rows_kernel<T, 256>), dim3((unsigned)R, (unsigned)B), dim3(256), 0, st, (const T*)logits, labels, off, nseq,
                       top, inv, lp, R, K);
}

template <typename T>
void pf_grad_launch(int B, int R, int K, int pairs, const void* logits, const int32_t* labels, const int32_t* off, const float* top,
                    const float* inv, const float* coef, const float* term, float* loss, void* dlogits, hipStream_t st) {
  if (pf_narrow(K, sizeof(T)))
    hipLaunchKernelGGL((pf_grad_kernel<T, 64>), dim3((unsigned)(R + 3) / 4 + 1u, (unsigned)B), dim3(256), 0, st, (const T*)logits, labels,
                       off, pairs, top, inv, coef, term, loss, (T*)dlogits, R, K);
  else
    hipLaunchKernelGGL((pf_grad_kernel<T, 256>), dim3((unsigned)R + 1u, (unsigned)B), dim3(256), 0, st, (const T*)logits, labels, off,
                       pairs, top, inv, coef, term, loss, (T*)dlogits, R, K);
}

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" {

int hfta_seq_logps(int B, int R, int K, int nseq, int dtype, const void* logits, const int32_t* labels, const int32_t* seq_offsets,
                   float* token_logps, float* logps, void* stream) {
  const int rc = pf_check(B, R, K, nseq, dtype);
  if (rc == HFTA_EINVAL || !logits || !labels || !seq_offsets || !token_logps || !logps) return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  hipStream_t st = as_stream(stream);
  if (dtype == HFTA_BF16) pf_rows_launch<bf16_raw>(B, R, K, nseq, logits, labels, seq_offsets, nullptr, nullptr, token_logps, st);
  else pf_rows_launch<float>(B, R, K, nseq, logits, labels, seq_offsets, nullptr, nullptr, token_logps, st);
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  hipLaunchKernelGGL(pf_seq_kernel, dim3((unsigned)nseq, (unsigned)B), dim3(256), 0, st, token_logps, seq_offsets, nseq,
                     logps, R);
  return launch_status();
}

size_t hfta_preference_loss_workspace_bytes(int B, int R, int npairs) {
  if (B <= 0 || R <= 0 || npairs <= 0 || npairs > PACKED_MAX / 2) return 0;
  return ((size_t)B * R * 4 + (size_t)B * npairs) * sizeof(float);     // largest value, inverse sum, label term and factor of the rows; pair terms
}

int hfta_preference_loss(int B, int R, int K, int npairs, int dtype, const void* logits, const int32_t* labels,
                         const int32_t* seq_offsets, const float* ref_logps, const float* beta, const float* label_smoothing,
                         float* loss, float* logps, void* dlogits, void* workspace, size_t ws_bytes, void* stream) {
  const int rc = pf_check(B, R, K, npairs > PACKED_MAX / 2 ? 0x7fffffff : npairs, dtype);
  if (rc == HFTA_EINVAL || !logits || !labels || !seq_offsets || !ref_logps || !beta || !loss || !logps || !dlogits)
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 4 || ws_bytes < hfta_preference_loss_workspace_bytes(B, R, npairs))
    return HFTA_EWORKSPACE;
  hipStream_t st = as_stream(stream);
  const size_t rows = (size_t)B * R;
  float *top = (float*)workspace, *inv = top + rows, *lp = inv + rows, *coef = lp + rows, *term = coef + rows;
  if (dtype == HFTA_BF16) pf_rows_launch<bf16_raw>(B, R, K, 2 * npairs, logits, labels, seq_offsets, top, inv, lp, st);
  else pf_rows_launch<float>(B, R, K, 2 * npairs, logits, labels, seq_offsets, top, inv, lp, st);
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  hipLaunchKernelGGL(pf_pair_kernel, dim3((unsigned)npairs, (unsigned)B), dim3(256), 0, st, lp, seq_offsets,
                     npairs, ref_logps, beta, label_smoothing, logps, term, coef, R);
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  if (dtype == HFTA_BF16)
    pf_grad_launch<bf16_raw>(B, R, K, npairs, logits, labels, seq_offsets, top, inv, coef, term, loss, dlogits, st);
  else
    pf_grad_launch<float>(B, R, K, npairs, logits, labels, seq_offsets, top, inv, coef, term, loss, dlogits, st);
  return launch_status();
}

}  // extern "C"
