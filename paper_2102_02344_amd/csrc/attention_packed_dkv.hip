// Attention over packed sequences: the backward kernel of the keys and values, over all heads of their group
// (attention_packed.h).
#include "attention_packed.h"

namespace hfta {
namespace {

// The tiles from which a workgroup's keys are seen: the last rows first, all heads of the group each, so that the
// workgroups of a sequence's keys read the same ones at the same time.  A workgroup takes every a.parts-th.  Places are kept and moved
// on, not computed anew: products of 64-bit strides were a thousand cycles a tile.
template <int ROWS> struct PkPlaceOf {
  int i0, head, group, di, dh;
  __device__ __forceinline__ PkPlaceOf(const PkArgs& a, int glo, int nt, int part) {
    group = a.Hq / a.Hkv;
    head = part % group;
    i0 = glo + (nt - 1 - part / group) * ROWS;
    di = a.parts / group * ROWS;
    dh = a.parts % group;
  }
  __device__ __forceinline__ bool next() {                       // whether past the last head
    head += dh;
    i0 -= di;
    const bool past = head >= group;
    if (past) { head -= group; i0 -= ROWS; }
    return past;
  }
};
template <typename T, int ROWS> struct PkWalk : PkPlaceOf<ROWS> {
  const T *q, *c;                  // the tile's first row
  int64_t srow;                    // of LSE and D
  int64_t qd[2], cd[2];            // a step, and what a step past the last head adds
  __device__ __forceinline__ PkWalk(const PkArgs& a, int b, int hq, int glo, int nt, int part) : PkPlaceOf<ROWS>(a, glo, nt, part) {
    const int64_t gr = this->group, di = this->di, dh = this->dh, i0 = this->i0;
    q = pk_at<T>(a.Q, a.qs, b, hq + this->head) + i0 * a.qs.r;
    c = pk_at<T>(a.dCTX, a.cs, b, hq + this->head) + i0 * a.cs.r;
    srow = ((int64_t)b * a.Hq + hq) * a.R;
    qd[0] = dh * a.qs.h - di * a.qs.r;
    cd[0] = dh * a.cs.h - di * a.cs.r;
    qd[1] = -gr * a.qs.h - ROWS * a.qs.r;
    cd[1] = -gr * a.cs.h - ROWS * a.cs.r;
  }
  __device__ __forceinline__ void next() {
    q += qd[0];
    c += cd[0];
    if (PkPlaceOf<ROWS>::next()) {
      q += qd[1];
      c += cd[1];
    }
  }
};

// The sums of 32 keys, their operands and the scores are more registers than two wavefronts per SIMD can have (heads of 128).  So
// two wavefronts share 32 keys: one forms p and dv, the other dctx . v, takes p from LDS, and forms ds and dk -- the same products,
// half the registers each.  Two barriers per 32 rows; a workgroup takes 64 keys.  Where workgroups are few or uneven (the first
// keys of a long sequence are seen by all its rows) a.parts of them share the tiles of 64 keys; their sums go through the workspace.
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256, (D * (int)sizeof(T) <= 128 ? 4 : D * (int)sizeof(T) <= 256 ? 3 : 2)) void pk_dkv_kernel(PkArgs a) {
  typedef PkStage<T, D, VEC, false, 32> Stage;
  constexpr int ROWS = 32, BM = 64, NBUF = 2;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[NBUF * 2 * Stage::BYTES];
  __shared__ __attribute__((aligned(16))) float stats[NBUF][2][ROWS];      // lse and D of the tile's rows
  __shared__ __attribute__((aligned(16))) float prob[2][4][64][4];         // p of a pair: as its wavefronts hold it
  __shared__ PackedRows<BM> pr;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const int pair = wave >> 1;
  const bool forms_v = (wave & 1) == 0;
  const PkPlace<BM, true> at(a);
  const int part = at.part;
  PkSpan<BM> sp;
  const int own = at.t0 + pair * PK_WT + (lane & 31);
  PkRow<T, D> x;                                                           // the first's keys, the second's values
  pk_load_row<T, D, VEC>(x, pk_at<T>(forms_v ? a.K : a.V, a.ks, at.b, at.hk) + (int64_t)own * a.ks.r, own < a.R, a.d, g);
  sp.template init<true>(pr, a, at.b, at.t0, pair * PK_WT);
  if (sp.glo >= sp.ghi) return;
  const float c = a.scale * PK_LOG2E;
  const int group = a.Hq / a.Hkv, nt = (sp.ghi - sp.glo + ROWS - 1) / ROWS, total = nt * group;
  pk_f16 o[D / 32];
  for (bool safe = false;; safe = true) {
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = pk_f16{};
    int buf = 0;
    Stage nq, nc;
    nq.init(a.qs.r, a.d);
    nc.init(a.cs.r, a.d);
    PkWalk<T, ROWS> w(a, at.b, at.hq, sp.glo, nt, part);
    auto place = [&](int b, int i) { return tiles + (b * 2 + i) * Stage::BYTES; };
    int nf = part;                                                         // the next tile that is loaded
    auto fetch = [&](int b) {
      const int rows = sp.ghi - w.i0;
      if (wave < 2) pk_fetch32(stats[b][wave], (wave ? a.Dsum : a.LSE) + w.srow + (int64_t)w.head * a.R + w.i0, rows, lane);
      nq.fetch(place(b, 0), w.q, a.qs.r, rows, a.d);
      nc.fetch(place(b, 1), w.c, a.cs.r, rows, a.d);
      w.next();
      nf += a.parts;
    };
    if (!safe && nf < total) fetch(buf);
    PkPlaceOf<ROWS> at_(a, sp.glo, nt, part);                              // first row of the tile that is multiplied
    for (int n = part; n < total; n += a.parts) {
      if (__builtin_expect(safe, 0)) {                                                          // one at a time
        __syncthreads();
        fetch(buf);
      }
      pk_landed();                                                         // lse and D
      nq.land(place(buf, 0));
      nc.land(place(buf, 1));
      __syncthreads();
      const int j0 = at_.i0;
      at_.next();
      if (!safe && nf < total) fetch(buf ^ 1);
      unsigned char* tq = place(buf, 0);
      unsigned char* tc = place(buf, 1);
      const bool some = !sp.none(j0, 32);
      pk_f16 sn[1] = {pk_f16{}};
      pk_f16& s = sn[0];
      if (some) {
        __builtin_amdgcn_s_setprio(1);
        pk_rows<T, D, 1>(sn, forms_v ? tq : tc, 0, x, lane);
        if constexpr (sizeof(T) == 2) pk_order<4, D / 16, 1>();
        __builtin_amdgcn_s_setprio(0);
        if (forms_v) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float4 ls = *reinterpret_cast<const float4*>(&stats[buf][0][y * 8 + 4 * g]);
            const float lv[4] = {ls.x, ls.y, ls.z, ls.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * y + e] = pk_exp2(fmaf(c, s[4 * y + e], -PK_LOG2E * lv[e]));
          }
          sp.mask(s, j0, g, 0.f);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            *reinterpret_cast<float4*>(prob[pair][y][lane]) = make_float4(s[4 * y], s[4 * y + 1], s[4 * y + 2], s[4 * y + 3]);
        }
      }
      __syncthreads();
      if (some && !forms_v) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float4 ds = *reinterpret_cast<const float4*>(&stats[buf][1][y * 8 + 4 * g]);
          const float4 p = *reinterpret_cast<const float4*>(prob[pair][y][lane]);
          const float dd[4] = {ds.x, ds.y, ds.z, ds.w}, pv[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * y + e] = pv[e] * (s[4 * y + e] - dd[e]);
        }
        sp.mask(s, j0, g, 0.f);
      }
      if (__builtin_expect(safe, 0)) {
        if (some) pk_mark<T, D>(o, forms_v ? tc : tq, 0, j0, sp.lo, sp.hi, lane);
        __syncthreads();
        Stage::clean(tq, ROWS);
        Stage::clean(tc, ROWS);
        __syncthreads();
      }
      if (some) {
        __builtin_amdgcn_s_setprio(1);
        pk_cols<T, D>(o, forms_v ? tc : tq, 0, s, lane);
        if constexpr (sizeof(T) == 2) pk_order<4, D / 16, 2>();
        __builtin_amdgcn_s_setprio(0);
      }
      if (!safe) buf ^= 1;
    }
    if (safe || !__syncthreads_or(sp.in && pk_not_finite(o))) break;
  }
  if (!sp.in) return;
  if (a.parts == 1) {
    T* row = pk_at<T>(forms_v ? a.dV : a.dK, a.dks, at.b, at.hk) + (int64_t)sp.row * a.dks.r;
    pk_store_row<T, D / 32, VEC>(row, o, forms_v ? 1.f : a.scale, 0, a.d, g);
  } else {                                                                 // [parts][dk, dv][B][Hkv][R][d]
    float* row = a.part + ((((int64_t)part * 2 + forms_v) * a.B + at.b) * a.Hkv + at.hk) * a.R * a.d + (int64_t)sp.row * a.d;
    pk_store_row<float, D / 32, VEC>(row, o, forms_v ? 1.f : a.scale, 0, a.d, g);
  }
}

// The parts' sums, added in order: a workgroup takes 32 rows of one key head, dk and dv.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void pk_parts_kernel(PkArgs a) {
  constexpr int ROWS = 32, W = VEC ? 4 : 1;
  __shared__ PackedRows<ROWS> pr;
  const int nk = a.B * a.Hkv, kh = blockIdx.x % nk, b = kh / a.Hkv, hk = kh % a.Hkv, t0 = blockIdx.x / nk * ROWS;
  pr.template scan<256>(a.off + (int64_t)b * (a.nseq + 1), a.nseq, a.R, t0);
  const int ppr = a.d / W, lo = max(t0, pr.first), hi = min(t0 + ROWS, pr.last);
  const int64_t all = (int64_t)nk * a.R * a.d;
  for (int i = threadIdx.x; i < (hi - lo) * 2 * ppr; i += 256) {
    const int c = i % ppr * W, x = i / ppr & 1, row = lo + i / ppr / 2;
    const float* src = a.part + x * all + ((int64_t)kh * a.R + row) * a.d + c;
    float y[PK_PARTS_MAX][W], v[W];
#pragma unroll
    for (int p = 0; p < PK_PARTS_MAX; ++p)                         // all in flight
      if (p < a.parts) {
        if constexpr (VEC) {
          const float4 f = *reinterpret_cast<const float4*>(src + 2 * p * all);
          y[p][0] = f.x; y[p][1] = f.y; y[p][2] = f.z; y[p][3] = f.w;
        } else {
          y[p][0] = src[2 * p * all];
        }
      }
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = y[0][e];
#pragma unroll
    for (int p = 1; p < PK_PARTS_MAX; ++p)
      if (p < a.parts) {
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] += y[p][e];
      }
    T* dst = pk_at<T>(x ? a.dV : a.dK, a.dks, b, hk) + (int64_t)row * a.dks.r + c;
    if constexpr (!VEC) Elem<T>::store(dst, v[0]);
    else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    else *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

template <typename T, int D> int launch(const PkArgs& a, const PkForm& f, hipStream_t st) {
  const dim3 grid((unsigned)(pk_tiles(a.R, 2 * PK_WT) * a.B * a.Hkv * a.parts)), block(256);
  if (f.vec) hipLaunchKernelGGL((pk_dkv_kernel<T, D, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((pk_dkv_kernel<T, D, false>), grid, block, 0, st, a);
  const int rc = launch_status();
  if (a.parts == 1 || rc != HFTA_OK) return rc;
  const dim3 gp((unsigned)(pk_tiles(a.R, 32) * a.B * a.Hkv));
  if (f.vec) hipLaunchKernelGGL((pk_parts_kernel<T, true>), gp, block, 0, st, a);
  else hipLaunchKernelGGL((pk_parts_kernel<T, false>), gp, block, 0, st, a);
  return launch_status();
}

}  // namespace

int pk_dkv(const PkArgs& a, const PkForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
