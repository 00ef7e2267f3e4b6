// Attention over packed sequences: the forward kernel (attention_packed.h).
#include "attention_packed.h"

namespace hfta {
namespace {

template <typename T, int D, bool VEC, bool SPLIT>
__global__ __launch_bounds__(256, (D * sizeof(T) <= 256 ? 2 : 1)) void pk_fwd_kernel(PkArgs a) {
  typedef PkStage<T, D, VEC, SPLIT> Stage;
  constexpr int NB = SPLIT ? 1 : 2, BM = pk_bm<SPLIT>();         // key blocks per tile, rows of the workgroup
  constexpr int NBUF = SPLIT ? 4 : 2;                            // tiles: a wavefront's, or in turn
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[NBUF * 2 * Stage::BYTES];
  __shared__ PackedRows<BM> pr;
  __shared__ float jm[4][32], jl[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const PkPlace<BM, false> at(a);
  PkSpan<BM> sp;
  const int row0 = SPLIT ? 0 : wave * PK_WT, own = at.t0 + row0 + (lane & 31);
  PkRow<T, D> q;                                                 // (what stands in rows of no sequence does not matter)
  pk_load_row<T, D, VEC>(q, pk_at<T>(a.Q, a.qs, at.b, at.hq) + (int64_t)own * a.qs.r, own < a.R, a.d, g);
  sp.template init<false>(pr, a, at.b, at.t0, row0);
  if (sp.glo >= sp.ghi) return;
  const T* kp = pk_at<T>(a.K, a.ks, at.b, at.hk);
  const T* vp = pk_at<T>(a.V, a.ks, at.b, at.hk);
  const float c = a.scale * PK_LOG2E;
  const int first = sp.glo + (SPLIT ? wave * 32 : 0);
  constexpr int STEP = SPLIT ? 128 : 64;
  pk_f16 o[D / 32];
  float m, l;
  for (bool safe = false;; safe = true) {
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = pk_f16{};
    m = -INFINITY;
    l = 0.f;
    int buf = SPLIT ? wave : 0;
    Stage nk, nv;
    nk.init(a.ks.r, a.d);
    nv.init(a.ks.r, a.d);
    const T *kt = kp + (int64_t)first * a.ks.r, *vt = vp + (int64_t)first * a.ks.r;
    const int64_t step = (int64_t)STEP * a.ks.r;
    int kf = first;                                              // the next tile that is loaded
    auto place = [&](int b, int i) { return tiles + (b * 2 + i) * Stage::BYTES; };
    auto fetch = [&](int b) {
      nk.fetch(place(b, 0), kt, a.ks.r, sp.ghi - kf, a.d);
      nv.fetch(place(b, 1), vt, a.ks.r, sp.ghi - kf, a.d);
      kt += step;
      vt += step;
      kf += STEP;
    };
    if (!safe && kf < sp.ghi) fetch(buf);
    for (int k0 = first; k0 < sp.ghi; k0 += STEP) {
      if (__builtin_expect(safe, 0)) {                                                // one at a time
        pk_sync<SPLIT>();
        fetch(buf);
      }
      nk.land(place(buf, 0));
      nv.land(place(buf, 1));
      pk_sync<SPLIT>();
      if (!safe && kf < sp.ghi) fetch(SPLIT ? buf : buf ^ 1);
      const unsigned char* tk = place(buf, 0);
      unsigned char* tv = place(buf, 1);
      const bool some = !sp.none(k0, NB * 32);
      pk_f16 s[NB];
      float mu = 0.f;
      if (some) {
        float mt = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) s[kb] = pk_f16{};
        __builtin_amdgcn_s_setprio(1);
        pk_rows<T, D, NB>(s, tk, 0, q, lane);
        if constexpr (sizeof(T) == 2) pk_order<4, NB * D / 16, 1>();
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) sp.mask(s[kb], k0 + kb * 32, g, -INFINITY);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[kb][i]);
        mt = pk_both_max(mt);
        // The maximum that p is taken against moves only where it would let p grow past 2^PK_SLACK: sums and products are
        // consistent with any, and are divided by each other at the end.  (Each row by itself: its bits do not depend on the others.)
        const bool grows = c * mt > m + PK_SLACK;
        if (__any(grows)) {
          const float f = grows ? pk_exp2(m - c * mt) : 1.f;
          l *= f;
#pragma unroll
          for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[n][i] *= f;
          m = grows ? c * mt : m;
        }
        mu = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            s[kb][i] = pk_exp2(fmaf(c, s[kb][i], -mu));
            l += s[kb][i];
          }
      }
      if (__builtin_expect(safe, 0)) {
        if (some) {
#pragma unroll
          for (int kb = 0; kb < NB; ++kb) pk_mark<T, D>(o, tv, kb * 32, k0 + kb * 32, sp.lo, sp.hi, lane);
        }
        pk_sync<SPLIT>();
        Stage::clean(tv, Stage::ROWS);
        pk_sync<SPLIT>();
      }
      if (some) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) pk_cols<T, D>(o, tv, kb * 32, s[kb], lane);
        if constexpr (sizeof(T) == 2) pk_order<4, NB * D / 16, 2>();
        __builtin_amdgcn_s_setprio(0);
      }
      if (!SPLIT && !safe) buf ^= 1;
    }
    if (safe || !__syncthreads_or(sp.in && pk_not_finite(o))) break;
  }
  l += __shfl_xor(l, 32, 64);
  if constexpr (SPLIT) {
    if (g == 0) { jm[wave][lane] = m; jl[wave][lane] = l; }
    __syncthreads();
    const int r = lane & 31;
    m = fmaxf(fmaxf(jm[0][r], jm[1][r]), fmaxf(jm[2][r], jm[3][r]));
    const float mu = m == -INFINITY ? 0.f : m, f = pk_exp2(jm[wave][r] - mu);
    l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) l += jl[w][r] * pk_exp2(jm[w][r] - mu);
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][i] *= f;
    pk_join<D>(o, reinterpret_cast<float*>(tiles), wave, lane);
    if (wave >= D / 32) return;
  }
  if (sp.in) {
    T* row = pk_at<T>(a.CTX, a.cs, at.b, at.hq) + (int64_t)sp.row * a.cs.r;
    if constexpr (SPLIT) {
      const pk_f16 one[1] = {o[0]};
      pk_store_row<T, 1, VEC>(row, one, 1.f / l, wave, a.d, g);
    } else {
      pk_store_row<T, D / 32, VEC>(row, o, 1.f / l, 0, a.d, g);
    }
    if (g == 0 && (!SPLIT || wave == 0)) a.LSE[((int64_t)at.b * a.Hq + at.hq) * a.R + sp.row] = (m + __builtin_amdgcn_logf(l)) * PK_LN2;
  }
}

template <typename T, int D> int launch(const PkArgs& a, const PkForm& f, hipStream_t st) {
  const dim3 grid((unsigned)(pk_tiles(a.R, f.split ? PK_WT : 4 * PK_WT) * a.B * a.Hq)), block(256);
  if (f.split) hipLaunchKernelGGL((pk_fwd_kernel<T, D, true, true>), grid, block, 0, st, a);
  else if (f.vec) hipLaunchKernelGGL((pk_fwd_kernel<T, D, true, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((pk_fwd_kernel<T, D, false, false>), grid, block, 0, st, a);
  return launch_status();
}

}  // namespace

int pk_fwd(const PkArgs& a, const PkForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
