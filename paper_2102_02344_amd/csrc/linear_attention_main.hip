// Linear attention: the walk over the tiles of a block (linear_attention.h).
#include "linear_attention.h"

namespace hfta {
namespace {

// of the wavefront's columns of c: NaN into the rows that see a value of the tile which is not finite
template <typename T, int D>
__device__ __forceinline__ void la_mark(pk_f16& acc, const unsigned char* tc, const LaWave<D>& wv, int tb, int rel) {
  const int t = 32 * tb + (wv.lane & 31);
#pragma unroll 1
  for (int r = 0; r < LA_T; ++r) {
    const bool sees = r >= rel && r <= t;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int c = 32 * wv.cs + 8 * (i >> 2) + 4 * wv.g + (i & 3);
      const float x = Elem<T>::load(reinterpret_cast<const T*>(tc + PkTile<T, D>::at(r, c * (int)sizeof(T)))), y = sees ? x : 0.f;
      acc[i] += y - y;                                           // NaN, or nothing
    }
  }
}

template <typename T, int D, bool VEC> __global__ __launch_bounds__(256, (D * sizeof(T) <= 256 ? 2 : 1)) void la_main_kernel(LaArgs a) {
  typedef LaStage<T, D, VEC> Stage;
  typedef PkTile<T, D> Tile;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int TH = LaWave<D>::TH, NTB = LaWave<D>::NTB;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[3 * Stage::BYTES], P[16384];
  __shared__ LaRows lr;
  __shared__ __attribute__((aligned(16))) float pw[LA_T + 1], wt[LA_T], fac[LA_T];
  unsigned char *ta = tiles, *tb = tiles + Stage::BYTES, *tc = tiles + 2 * Stage::BYTES;
  const LaWave<D> wv;
  const int lane = wv.lane, g = wv.g, t = threadIdx.x;
  const LaPlace at(a, false);
  const LaJob& J = a.job[at.job];
  const int rev = J.rev, hk = at.h / J.ga;
  const int32_t* off = a.off + (int64_t)at.b * (a.nseq + 1);
  const float ld = la_decay(a.ld[(int64_t)at.b * a.Hkv + hk]);
  if (t <= LA_T) pw[t] = la_pow(ld, t);
  const int first = at.blk * a.per, last = min(first + a.per, a.tiles) - 1;
  const bool keeps = J.S1 && at.h % J.ga == 0, pieces = J.S0 || keeps;

  if (keeps)                                                     // sequences without rows
    for (int s0 = at.blk * 256; s0 < a.nseq; s0 += a.blocks * 256) {
      const int s = s0 + t, lo = s < a.nseq ? min(max(off[s], 0), a.R) : 0, hi = s < a.nseq ? min(max(off[s + 1], 0), a.R) : 1;
      uint64_t m = __ballot(lo >= hi);
      for (; m; m &= m - 1) {
        const int64_t p = la_state_at<T, D>(a, at.b, s0 + wv.wave * 64 + __builtin_ctzll(m), hk);
        for (int i = lane; i < a.d * a.d; i += 64) J.S1[p + i] = J.S0 ? J.S0[p + i] : 0.f;
      }
    }

  // the block of 32 x 32 products that this wavefront forms, and the decays between its rows
  const int qt = TH == 1 ? wv.wave > 0 : wv.th & 1, qs = TH == 1 ? wv.wave == 2 : D == 64 ? wv.cs : wv.th >> 1;
  const bool forms = TH == 1 ? wv.wave < 3 : qt >= qs, sums = TH < 4 || wv.th < 2;
  const int tb0 = TH == 1 ? 0 : wv.th & 1;                       // first of its NTB blocks of rows
  __syncthreads();
  pk_f16 D0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = 32 * (qt - qs) + (lane & 31) - (8 * (i >> 2) + 4 * g + (i & 3));
    D0[i] = n >= 0 ? pw[n] : 0.f;
  }

  pk_f16 s[D / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n) s[n] = pk_f16{};
  const T* pa = pk_at<T>(J.A, J.as, at.b, at.h);
  const T* pb = pk_at<T>(J.B, J.bs, at.b, 0);
  const T* pc = pk_at<T>(J.C, J.cs, at.b, 0);
  T* po = pk_at<T>(J.O, J.os, at.b, at.h);

  for (int tile = first; tile <= last; ++tile) {
    const int m0 = (rev ? a.tiles - 1 - tile : tile) * LA_T;
    __syncthreads();
    la_rows(lr, off, a, rev, tile, (tile - first) % (LA_SPAN / LA_T) == 0);
    const int mine = lr.rel[lane];
    if (tile == first && tile > 0 && lr.rel[0] == -1) {          // the state that the first row's sequence brings from the blocks before
      int start, end;
      const int r = rev ? m0 + LA_T - 1 : m0;
      lr.pr.range(lr.t0, r - lr.t0, start, end);
      const int begin = rev ? a.tiles * LA_T - end : start;
      const float* sum = a.sums + (((int64_t)at.job * a.B + at.b) * a.Hkv + hk) * a.blocks * (D * D);
      const float m1 = la_powm1(ld, a.per * LA_T);
      for (int k = a.scanned ? at.blk - 1 : begin / (a.per * LA_T); k < at.blk; ++k) {
        la_fade(s, m1);
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 v = *la_sum<D>(const_cast<float*>(sum) + (int64_t)k * (D * D), wv.cs, n, q, lane);
            s[n][4 * q] += v.x;
            s[n][4 * q + 1] += v.y;
            s[n][4 * q + 2] += v.z;
            s[n][4 * q + 3] += v.w;
          }
      }
    }
    const uint64_t there = __ballot(mine != LA_NONE);
    if (!there) continue;
    // all rows at once, or where states come in or go out one sequence after another
    for (int p0 = pieces ? __builtin_ctzll(there) : 0, p1; p0 < LA_T;) {
      const int val = __builtin_amdgcn_readlane(mine, pieces ? p0 : LA_T - 1);
      const bool begins = pieces && val >= 0;
      p1 = LA_T;
      if (pieces) {
        const uint64_t m = __ballot(mine != val && lane > p0);
        if (m) p1 = __builtin_ctzll(m);
      }
      // rows of the state's product and of its update, and how far the state fades
      const int c0 = pieces ? p0 : val == LA_NONE ? LA_T : max(val, 0), late = begins && J.S0 && rev ? 1 : 0;
      if (begins) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) s[n] = pk_f16{};
        if (J.S0) {
          int lo = 0, n = a.nseq;                                // the last sequence that begins at or before the row
          const int r = rev ? m0 + LA_T - 1 - p0 : m0 + p0;
          while (n > 1) {
            const int half = n >> 1;
            if (off[lo + half] <= r) { lo += half; n -= half; } else n = half;
          }
          la_load_state<T, D>(s, J, a, at.b, lo, hk, wv);
        }
      }
      const bool brings = pieces ? !begins || J.S0 : __builtin_amdgcn_readlane(mine, 0) == -1;
      const bool ends = keeps && lr.seqend[p1 - 1], updates = pieces ? ends || (p1 == LA_T && tile < last) : c0 < LA_T && tile < last;
      pk_f16 acc[NTB];
#pragma unroll
      for (int n = 0; n < NTB; ++n) acc[n] = pk_f16{};
      for (int h = 0; h < J.gb; ++h) {
        const int hb = at.h / J.ga * J.gb + h;
        __syncthreads();                                         // what the last pass reads has been read
        if (t < LA_T) {
          wt[t] = t >= c0 && t < p1 ? pw[p1 - 1 - t] : 0.f;
          fac[t] = pieces ? (t >= p0 && t < p1 ? pw[t - p0 + 1 - late] : 0.f) : lr.rel[t] == -1 ? pw[t + 1] : 0.f;
        }
        if (h == 0) Stage::fetch(ta, pa + (int64_t)m0 * J.as.r, J.as.r, a.R - m0, a.d, rev);
        Stage::fetch(tb, pb + hb * J.bs.h + (int64_t)m0 * J.bs.r, J.bs.r, a.R - m0, a.d, rev);
        Stage::fetch(tc, pc + hb * J.cs.h + (int64_t)m0 * J.cs.r, J.cs.r, a.R - m0, a.d, rev);
        la_land<VEC>();
#pragma unroll
        for (int n = 0; n < NTB; ++n) {
          const int blk = tb0 + n;
          const bool product = forms && qt == blk, inter = sums && brings && h == 0;
          if (!product && !inter) continue;
          PkRow<T, D> x;
#pragma unroll
          for (int i = 0; i < PkRow<T, D>::N; ++i)
            x.p[i].u = *reinterpret_cast<const uint4*>(ta + Tile::at(32 * blk + (lane & 31), i * 32 + g * 16));
          if (product) {
            pk_f16 y[1] = {pk_f16{}};
            pk_rows<T, D, 1>(y, tb, 32 * qs, x, lane);
            const int rel = lr.rel[32 * blk + (lane & 31)] - 32 * qs - 4 * g, self = 32 * (qt - qs) + (lane & 31) - 4 * g;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int r = 8 * (i >> 2) + (i & 3);
              y[0][i] = r >= rel && r <= self ? y[0][i] * D0[i] : 0.f;
            }
            if constexpr (BF) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                LaFrag hi, lo;
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                  const float x0 = y[0][8 * k + 2 * p], x1 = y[0][8 * k + 2 * p + 1];
                  hi.u[p] = pack_bf16x2(x0, x1);
                  lo.u[p] = pack_bf16x2(x0 - __uint_as_float(hi.u[p] << 16), x1 - __uint_as_float(hi.u[p] & 0xffff0000u));
                }
                const int to = PkTile<bf16_raw, 64>::at(32 * qt + (lane & 31), (2 * qs + k) * 32 + g * 16);
                *reinterpret_cast<uint4*>(P + to) = make_uint4(hi.u[0], hi.u[1], hi.u[2], hi.u[3]);
                *reinterpret_cast<uint4*>(P + 8192 + to) = make_uint4(lo.u[0], lo.u[1], lo.u[2], lo.u[3]);
              }
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4*>(P + PkTile<float, 64>::at(32 * qt + (lane & 31), (32 * qs + 8 * q + 4 * g) * 4)) =
                    make_float4(y[0][4 * q], y[0][4 * q + 1], y[0][4 * q + 2], y[0][4 * q + 3]);
            }
          }
          if (inter) {
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) {
              if constexpr (BF) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  LaFrag hi, lo;
#pragma unroll
                  for (int p = 0; p < 4; ++p) {
                    const float x0 = s[kb][8 * k + 2 * p], x1 = s[kb][8 * k + 2 * p + 1];
                    hi.u[p] = pack_bf16x2(x0, x1);
                    lo.u[p] = pack_bf16x2(x0 - __uint_as_float(hi.u[p] << 16), x1 - __uint_as_float(hi.u[p] & 0xffff0000u));
                  }
                  acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi.v, x.p[2 * kb + k].v, acc[n], 0, 0, 0);
                  acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo.v, x.p[2 * kb + k].v, acc[n], 0, 0, 0);
                }
              } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(s[kb][i], x.p[4 * kb + (i >> 2)].e[i & 3], acc[n], 0, 0, 0);
              }
            }
            const float f = fac[32 * blk + (lane & 31)];
            const bool sees = pieces ? 32 * blk + (lane & 31) >= p0 && 32 * blk + (lane & 31) < p1 : lr.rel[32 * blk + (lane & 31)] == -1;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][i] = sees ? f * acc[n][i] : 0.f;
          }
        }
        __syncthreads();
        if (sums) {                                              // the masked products with c
          if constexpr (BF) {
            LaFrag c[4];
            uint32_t odd = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              la_cols<D, false>(c[k], tc, 16 * k, 32 * wv.cs, lane);
#pragma unroll
              for (int p = 0; p < 4; ++p) odd |= la_odd(c[k].u[p]);
            }
            const bool marks = __any(odd & 0x80008000u);
            if (__builtin_expect(marks, 0)) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                  const uint32_t o = la_odd(c[k].u[p]);
                  c[k].u[p] &= (o & 0x8000u ? 0u : 0xffffu) | (o & 0x80000000u ? 0u : 0xffff0000u);
                }
            }
#pragma unroll
            for (int n = 0; n < NTB; ++n) {
              const int row = 32 * (tb0 + n) + (lane & 31);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (k >= 2 && tb0 + n == 0) continue;
                LaFrag hi, lo;
                const int from = PkTile<bf16_raw, 64>::at(row, k * 32 + g * 16);
                const uint4 vh = *reinterpret_cast<const uint4*>(P + from), vl = *reinterpret_cast<const uint4*>(P + 8192 + from);
                hi.u[0] = vh.x; hi.u[1] = vh.y; hi.u[2] = vh.z; hi.u[3] = vh.w;
                lo.u[0] = vl.x; lo.u[1] = vl.y; lo.u[2] = vl.z; lo.u[3] = vl.w;
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[k].v, hi.v, acc[n], 0, 0, 0);
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[k].v, lo.v, acc[n], 0, 0, 0);
              }
              if (__builtin_expect(marks, 0)) la_mark<T, D>(acc[n], tc, wv, tb0 + n, lr.rel[row]);
            }
          } else {
            float z = 0.f;
#pragma unroll 8
            for (int i = 0; i < 32; ++i)
              z = fmaf(0.f, *reinterpret_cast<const float*>(tc + Tile::at(2 * i + g, (32 * wv.cs + (lane & 31)) * 4)), z);
            const bool marks = __any(z != z);
#pragma unroll
            for (int n = 0; n < NTB; ++n) {
              const int row = 32 * (tb0 + n) + (lane & 31);
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                if (q >= 4 && tb0 + n == 0) continue;
                const float4 v = *reinterpret_cast<const float4*>(P + PkTile<float, 64>::at(row, (8 * q + 4 * g) * 4));
                const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float c = *reinterpret_cast<const float*>(tc + Tile::at(8 * q + 4 * g + e, (32 * wv.cs + (lane & 31)) * 4));
                  if (__builtin_expect(marks, 0) && (__float_as_uint(c) & 0x7f800000u) == 0x7f800000u) c = 0.f;
                  acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(c, w[e], acc[n], 0, 0, 0);
                }
              }
              if (__builtin_expect(marks, 0)) la_mark<T, D>(acc[n], tc, wv, tb0 + n, lr.rel[row]);
            }
          }
          if (h == J.gb - 1) {
#pragma unroll
            for (int n = 0; n < NTB; ++n) {
              const int j = 32 * (tb0 + n) + (lane & 31);
              if (lr.rel[j] == LA_NONE || j < p0 || j >= p1) continue;
              const pk_f16 one[1] = {acc[n]};
              pk_store_row<T, 1, VEC>(po + (int64_t)(rev ? m0 + LA_T - 1 - j : m0 + j) * J.os.r, one, J.fo, wv.cs, a.d, g);
            }
          }
        }
        if (updates && sums) {
          if (h == 0) {
            if (!pieces && val >= 0) {                            // a sequence that began in this tile
#pragma unroll
              for (int n = 0; n < D / 32; ++n) s[n] = pk_f16{};
            } else {
              la_fade(s, la_powm1(ld, p1 - c0 - late));
            }
          }
          la_update<T, D, 1>(s, tb, tc, wt, c0, p1, c0 > 0 || p1 < LA_T, J.S1 != nullptr, wv, 0);
        }
      }
      if (ends && (TH == 1 || wv.th == 0)) {
        int lo = 0, n = a.nseq;
        const int r = rev ? m0 + LA_T - p1 : m0 + p1 - 1;
        while (n > 1) {
          const int half = n >> 1;
          if (off[lo + half] <= r) { lo += half; n -= half; } else n = half;
        }
        float* out = J.S1 + la_state_at<T, D>(a, at.b, lo, hk);
        const int col = 32 * wv.cs + (lane & 31);
        const float f = J.fi * (rev ? pw[1] : 1.f);
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = 32 * k + la_row<T>(i, g);
            if (row < a.d && col < a.d) out[row * a.d + col] = f * s[k][i];
          }
      }
      if (!pieces) break;
      const uint64_t rest = p1 < LA_T ? there >> p1 << p1 : 0;
      p0 = rest ? __builtin_ctzll(rest) : LA_T;
    }
  }
}

template <typename T, int D> int launch(const LaArgs& a, const LaForm& f, hipStream_t st) {
  int64_t n = 0;
  for (int j = 0; j < a.jobs; ++j) n += (int64_t)a.blocks * a.B * a.job[j].heads;
  const dim3 grid((unsigned)n), block(256);
  if (f.vec) hipLaunchKernelGGL((la_main_kernel<T, D, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((la_main_kernel<T, D, false>), grid, block, 0, st, a);
  return launch_status();
}

}  // namespace

int la_main(const LaArgs& a, const LaForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
