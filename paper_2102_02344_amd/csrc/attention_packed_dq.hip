// Attention over packed sequences: the backward kernel of the queries, which also leaves D for the one of the keys
// (attention_packed.h).
#include "attention_packed.h"

namespace hfta {
namespace {

// p and ds are rounded to bf16 before their products, which leaves the gradients sqrt(2) of the error that rounding the results has by
// itself.  D from the stored ctx would add as much again as ctx's rounding is large against D, most where sequences are short.  What it
// lacks is in the sums anyway: with ds formed from D0, delta_i = sum_j ds_ij = D_i - D0_i.  The kernel of the keys gets D0 + delta.  Here
// dq_i lacks -delta_i sum_j p_ij k_j; where sequences are short (a.twice) delta is summed first, in a pass of its own that leaves
// out the product over keys.  Mean error of the three gradients in roundings of the results, 12 to 48 rows a sequence: 1.44 to 1.56 with
// neither, 1.40 to 1.51 with delta for the keys alone, 1.34 to 1.44 with both; 140 to 1000 rows: 1.41 to 1.46 with the first.
template <typename T, int D, bool VEC, bool SPLIT>
__global__ __launch_bounds__(256, (D * sizeof(T) <= 256 ? 2 : 1)) void pk_dq_kernel(PkArgs a) {
  constexpr bool FIX = sizeof(T) == 2;                           // (fp32 needs none of it)
  typedef PkStage<T, D, VEC, SPLIT> Stage;
  constexpr int NB = SPLIT ? 1 : 2, BM = pk_bm<SPLIT>();         // key blocks per tile, rows of the workgroup
  constexpr int NBUF = SPLIT ? 4 : 2;                            // tiles: a wavefront's, or in turn
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[NBUF * 2 * Stage::BYTES];
  __shared__ PackedRows<BM> pr;
  __shared__ float jd[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const PkPlace<BM, false> at(a);
  PkSpan<BM> sp;
  const int row0 = SPLIT ? 0 : wave * PK_WT, own = at.t0 + row0 + (lane & 31);
  const bool there = own < a.R;                                  // (what stands in rows of no sequence does not matter)
  const int64_t srow = ((int64_t)at.b * a.Hq + at.hq) * a.R + own;
  PkRow<T, D> q, dc;
  float lse, dsum = 0.f;
  {
    PkRow<T, D> x;
    pk_load_row<T, D, VEC>(dc, pk_at<T>(a.dCTX, a.cs, at.b, at.hq) + (int64_t)own * a.cs.r, there, a.d, g);
    pk_load_row<T, D, VEC>(x, pk_at<T>(a.CTX, a.cs, at.b, at.hq) + (int64_t)own * a.cs.r, there, a.d, g);
    pk_load_row<T, D, VEC>(q, pk_at<T>(a.Q, a.qs, at.b, at.hq) + (int64_t)own * a.qs.r, there, a.d, g);
    lse = there ? a.LSE[srow] : 0.f;
    sp.template init<false>(pr, a, at.b, at.t0, row0);
    if (sp.glo >= sp.ghi) return;
#pragma unroll
    for (int s = 0; s < PkRow<T, D>::N; ++s)
#pragma unroll
      for (int e = 0; e < PkRow<T, D>::EPP; ++e) dsum = fmaf(Elem<T>::to_f32(x.p[s].e[e]), Elem<T>::to_f32(dc.p[s].e[e]), dsum);
    dsum += __shfl_xor(dsum, 32, 64);
  }
  lse *= PK_LOG2E;
  const T* kp = pk_at<T>(a.K, a.ks, at.b, at.hk);
  const T* vp = pk_at<T>(a.V, a.ks, at.b, at.hk);
  const float c = a.scale * PK_LOG2E;
  const int first = sp.glo + (SPLIT ? wave * 32 : 0);
  constexpr int STEP = SPLIT ? 128 : 64;
  pk_f16 o[D / 32];
  float delta;
  for (int pass = FIX && a.twice ? 0 : 1;; ++pass) {
    const bool sums = FIX && pass == 0, safe = pass == 2;        // delta alone; values that are not finite
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = pk_f16{};
    delta = 0.f;
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
      unsigned char* tk = place(buf, 0);
      const unsigned char* tv = place(buf, 1);
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const int j0 = k0 + kb * 32;
        const bool some = !sp.none(j0, 32);
        pk_f16 s[1] = {pk_f16{}};
        if (some) {
          pk_f16 p[1] = {pk_f16{}};
          pk_rows<T, D, 1>(s, tk, kb * 32, q, lane);
          pk_rows<T, D, 1>(p, tv, kb * 32, dc, lane);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[0][i] = pk_exp2(fmaf(c, s[0][i], -lse)) * (p[0][i] - dsum);
          sp.mask(s[0], j0, g, 0.f);
          if constexpr (FIX)
#pragma unroll
            for (int i = 0; i < 16; ++i) delta += s[0][i];
        }
        if (__builtin_expect(safe, 0)) {
          if (some) pk_mark<T, D>(o, tk, kb * 32, j0, sp.lo, sp.hi, lane);
          pk_sync<SPLIT>();
          Stage::clean(tk + kb * 32 * PkTile<T, D>::ROW, 32);
          pk_sync<SPLIT>();
        }
        if (some && !sums) pk_cols<T, D>(o, tk, kb * 32, s[0], lane);
      }
      if (!SPLIT && !safe) buf ^= 1;
    }
    if constexpr (FIX) {                                         // (a second time: what the sums still lack)
      delta += __shfl_xor(delta, 32, 64);
      if constexpr (SPLIT) {
        if (g == 0) jd[wave][lane] = delta;
        __syncthreads();
        delta = (jd[0][lane & 31] + jd[1][lane & 31]) + (jd[2][lane & 31] + jd[3][lane & 31]);
      }
      if (sums) {
        dsum += delta;
        __syncthreads();
        continue;
      }
    }
    if (safe || !__syncthreads_or(sp.in && pk_not_finite(o))) break;
  }
  if constexpr (FIX) dsum += delta;
  if (sp.in && g == 0 && (!SPLIT || wave == 0)) a.Dsum[srow] = dsum;
  if constexpr (SPLIT) {
    pk_join<D>(o, reinterpret_cast<float*>(tiles), wave, lane);
    if (wave >= D / 32) return;
  }
  if (sp.in) {
    T* row = pk_at<T>(a.dQ, a.dqs, at.b, at.hq) + (int64_t)sp.row * a.dqs.r;
    if constexpr (SPLIT) {
      const pk_f16 one[1] = {o[0]};
      pk_store_row<T, 1, VEC>(row, one, a.scale, wave, a.d, g);
    } else {
      pk_store_row<T, D / 32, VEC>(row, o, a.scale, 0, a.d, g);
    }
  }
}

template <typename T, int D> int launch(const PkArgs& a, const PkForm& f, hipStream_t st) {
  const dim3 grid((unsigned)(pk_tiles(a.R, f.split ? PK_WT : 4 * PK_WT) * a.B * a.Hq)), block(256);
  if (f.split) hipLaunchKernelGGL((pk_dq_kernel<T, D, true, true>), grid, block, 0, st, a);
  else if (f.vec) hipLaunchKernelGGL((pk_dq_kernel<T, D, true, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((pk_dq_kernel<T, D, false, false>), grid, block, 0, st, a);
  return launch_status();
}

}  // namespace

int pk_dq(const PkArgs& a, const PkForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
