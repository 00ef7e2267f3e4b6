// Attention over packed sequences: the backward kernel of the keys and values, over all heads of their group
// (attention_packed.h).
#include "attention_packed.h"

namespace hfta {
namespace {

template <typename T, int D, bool VEC, bool SPLIT>
__global__ __launch_bounds__(256, (D * sizeof(T) <= 128 ? 2 : 1)) void pk_dkv_kernel(PkArgs a) {
  typedef PkStage<T, D, VEC, SPLIT> Stage;
  constexpr int ROWS = Stage::ROWS, NB = ROWS / 32, NBUF = SPLIT ? 4 : 2, BM = pk_bm<SPLIT>();
  __shared__ __attribute__((aligned(16))) unsigned char tiles[NBUF * 2 * Stage::BYTES];
  __shared__ __attribute__((aligned(16))) float stats[NBUF][2][ROWS];      // lse and D of the tile's rows
  __shared__ PackedRows<BM> pr;
  __shared__ int lim[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const PkPlace<BM, true> at(a);
  PkSpan<BM> sp;
  sp.template init<true>(pr, lim, a, at.b, at.t0, SPLIT ? 0 : wave * PK_WT);
  if (sp.glo >= sp.ghi) return;
  PkRow<T, D> k, v;
  pk_load_row<T, D, VEC>(k, pk_at<T>(a.K, a.ks, at.b, at.hk) + (int64_t)sp.row * a.ks.r, sp.in, a.d, g);
  pk_load_row<T, D, VEC>(v, pk_at<T>(a.V, a.ks, at.b, at.hk) + (int64_t)sp.row * a.ks.r, sp.in, a.d, g);
  const float c = a.scale * PK_LOG2E;
  const int nt = (sp.ghi - sp.glo + ROWS - 1) / ROWS, total = nt * (a.Hq / a.Hkv);      // tiles of a head, of the group
  constexpr int STEP = SPLIT ? 4 : 1;
  pk_f16 dk[D / 32], dv[D / 32];
  for (bool safe = false;; safe = true) {
#pragma unroll
    for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = pk_f16{};
    int buf = SPLIT ? wave : 0;
    Stage nq, nc;
    float nl = 0.f;
    auto fetch = [&](int n) {
      const int h = at.hq + n / nt, i0 = sp.glo + n % nt * ROWS;
      nq.load(pk_at<T>(a.Q, a.qs, at.b, h), a.qs.r, i0, sp.ghi, a.d);
      nc.load(pk_at<T>(a.dCTX, a.cs, at.b, h), a.cs.r, i0, sp.ghi, a.d);
      if (Stage::tid() < 2 * ROWS) {
        const int i = i0 + Stage::tid() % ROWS;
        const int64_t at_ = ((int64_t)at.b * a.Hq + h) * a.R + i;
        nl = i < sp.ghi ? (Stage::tid() < ROWS ? a.LSE[at_] * PK_LOG2E : a.Dsum[at_]) : 0.f;
      }
    };
    auto put = [&] {
      nq.store(tiles + buf * 2 * Stage::BYTES);
      nc.store(tiles + (buf * 2 + 1) * Stage::BYTES);
      if (Stage::tid() < 2 * ROWS) (&stats[buf][0][0])[Stage::tid()] = nl;
    };
    const int first = SPLIT ? wave : 0;
    if (first < total) {
      fetch(first);
      put();
    }
    for (int n = first; n < total; n += STEP) {
      pk_sync<SPLIT>();
      const bool more = n + STEP < total;
      if (more && !safe) fetch(n + STEP);
      unsigned char* tq = tiles + buf * 2 * Stage::BYTES;
      unsigned char* tc = tiles + (buf * 2 + 1) * Stage::BYTES;
      const int i0 = sp.glo + n % nt * ROWS;
      pk_f16 s[NB], p[NB];
#pragma unroll
      for (int qb = 0; qb < NB; ++qb) {
        const int j0 = i0 + qb * 32;
        if (sp.none(j0, 32)) continue;
        s[qb] = pk_f16{};
        p[qb] = pk_f16{};
        pk_rows<D>(s[qb], tq, qb * 32, k, lane);
        pk_rows<D>(p[qb], tc, qb * 32, v, lane);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float4 ls = *reinterpret_cast<const float4*>(&stats[buf][0][qb * 32 + x * 8 + 4 * g]);
          const float4 ds = *reinterpret_cast<const float4*>(&stats[buf][1][qb * 32 + x * 8 + 4 * g]);
          const float lv[4] = {ls.x, ls.y, ls.z, ls.w}, dd[4] = {ds.x, ds.y, ds.z, ds.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * x + e;
            s[qb][i] = pk_exp2(fmaf(c, s[qb][i], -lv[e]));
            p[qb][i] = s[qb][i] * (p[qb][i] - dd[e]);
          }
        }
        if (!sp.all(j0, 32)) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!sp.sees(j0, i, g)) s[qb][i] = p[qb][i] = 0.f;
        }
        if (!safe) {
          pk_cols<T, D>(dv, tc, qb * 32, s[qb], lane);
          pk_cols<T, D>(dk, tq, qb * 32, p[qb], lane);
        }
      }
      if (safe) {
#pragma unroll
        for (int qb = 0; qb < NB; ++qb)
          if (!sp.none(i0 + qb * 32, 32)) {
            pk_mark<T, D>(dv, tc, qb * 32, i0 + qb * 32, sp.lo, sp.hi, lane);
            pk_mark<T, D>(dk, tq, qb * 32, i0 + qb * 32, sp.lo, sp.hi, lane);
          }
        pk_sync<SPLIT>();
        nq.clean();
        nc.clean();
        nq.store(tq);
        nc.store(tc);
        pk_sync<SPLIT>();
#pragma unroll
        for (int qb = 0; qb < NB; ++qb)
          if (!sp.none(i0 + qb * 32, 32)) {
            pk_cols<T, D>(dv, tc, qb * 32, s[qb], lane);
            pk_cols<T, D>(dk, tq, qb * 32, p[qb], lane);
          }
      }
      if (more) {
        if (safe) fetch(n + STEP);
        if (!SPLIT) buf ^= 1;
        pk_sync<true>();
        put();
      }
    }
    if (safe || !__syncthreads_or(sp.in && (pk_not_finite(dk) || pk_not_finite(dv)))) break;
  }
  if constexpr (SPLIT) {
    pk_join<D>(dk, reinterpret_cast<float*>(tiles), wave, lane);
    pk_join<D>(dv, reinterpret_cast<float*>(tiles), wave, lane);
    if (wave >= D / 32) return;
  }
  if (sp.in) {
    T* rk = pk_at<T>(a.dK, a.dks, at.b, at.hk) + (int64_t)sp.row * a.dks.r;
    T* rv = pk_at<T>(a.dV, a.dks, at.b, at.hk) + (int64_t)sp.row * a.dks.r;
    if constexpr (SPLIT) {
      const pk_f16 one[2][1] = {{dk[0]}, {dv[0]}};
      pk_store_row<T, 1, VEC>(rk, one[0], a.scale, wave, a.d, g);
      pk_store_row<T, 1, VEC>(rv, one[1], 1.f, wave, a.d, g);
    } else {
      pk_store_row<T, D / 32, VEC>(rk, dk, a.scale, 0, a.d, g);
      pk_store_row<T, D / 32, VEC>(rv, dv, 1.f, 0, a.d, g);
    }
  }
}

}  // namespace

int pk_dkv(const PkArgs& a, const PkForm& f, hipStream_t st) {
  PK_LAUNCH(pk_dkv_kernel, pk_tiles(a.R, f.split ? PK_WT : 4 * PK_WT) * a.B * a.Hkv);
}

}  // namespace hfta
