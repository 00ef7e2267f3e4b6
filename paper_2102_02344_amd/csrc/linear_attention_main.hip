// Linear attention: the walk over the tiles of a block (linear_attention.h).
#include "linear_attention.h"

namespace hfta {
namespace {

// of the wavefront's columns of c: NaN into the rows that see a value of the tile which is not finite
template <typename T, int D, int NTB>
__device__ __forceinline__ void la_mark(pk_f16 (&acc)[NTB], const unsigned char* tc, const LaWave<D>& wv, int tb0, const int* rel) {
  int c0 = 32 * wv.cs + 4 * wv.g;
  asm volatile("" : "+v"(c0));                                   // (nothing of this is worth a register outside)
#pragma unroll
  for (int n = 0; n < NTB; ++n) {
    const int t = 32 * (tb0 + n) + (wv.lane & 31), begin = rel[t];
#pragma unroll 1
    for (int r = 0; r < LA_T; ++r) {
      const bool sees = r >= begin && r <= t;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = c0 + 8 * (i >> 2) + (i & 3);
        const float x = Elem<T>::load(reinterpret_cast<const T*>(tc + PkTile<T, D>::at(r, c * (int)sizeof(T)))), y = sees ? x : 0.f;
        acc[n][i] += y - y;                                      // NaN, or nothing
      }
    }
  }
}

// a sequence's state from and to memory, and which sequence a row belongs to: the last one that begins at or before it
__device__ __forceinline__ int la_sequence(const int32_t* off, int nseq, int r) {
  int lo = 0;
  for (int n = nseq; n > 1;) {
    const int half = n >> 1;
    if (off[lo + half] <= r) { lo += half; n -= half; } else n = half;
  }
  return lo;
}
template <typename T, int D>
__device__ __forceinline__ void la_store_state(const pk_f16 (&s)[D / 32], float* p, int d, float f, const LaWave<D>& wv) {
  int col = 32 * wv.cs + (wv.lane & 31);
  asm volatile("" : "+v"(col));
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = 32 * k + la_row<T>(i, wv.g);
      if (row < d && col < d) p[row * d + col] = f * s[k][i];
    }
}

// PIECES: states come in or go out, and a tile is walked one sequence after another; otherwise it is taken at once
template <typename T, int D, bool VEC, bool PIECES> __global__ __launch_bounds__(256, (D * sizeof(T) <= 256 ? 2 : 1)) void la_main_kernel(LaArgs a) {
  typedef LaStage<T, D, VEC> Stage;
  typedef PkTile<T, D> Tile;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int TH = LaWave<D>::TH, NTB = LaWave<D>::NTB, ROW = Tile::ROW;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[3 * Stage::BYTES], P[16384];
  __shared__ LaRows lr;
  __shared__ __attribute__((aligned(16))) float pw[LA_T + 1], wt[LA_T], fac[LA_T];
  unsigned char *const ta = tiles, *const tb = tiles + Stage::BYTES, *const tc = tiles + 2 * Stage::BYTES;
  const la_lds la = (la_lds)tiles, lb = (la_lds)tiles + Stage::BYTES, lc = (la_lds)tiles + 2 * Stage::BYTES;
  const LaWave<D> wv;
  const int lane = wv.lane, g = wv.g, t = threadIdx.x;
  const LaPlace at(a, false);
  const LaJob& J = a.job[at.job];
  const int rev = J.rev, hk = at.h / J.ga, G = J.gb;
  const int32_t* off = a.off + (int64_t)at.b * (a.nseq + 1);
  const float ld = la_decay(a.ld[(int64_t)at.b * a.Hkv + hk]);
  if (t <= LA_T) pw[t] = la_pow(ld, t);
  const int first = at.blk * a.per, last = min(first + a.per, a.tiles) - 1;
  const bool keeps = PIECES && J.S1 && at.h % J.ga == 0;

  if constexpr (PIECES) {
    if (keeps)                                                   // sequences without rows
      for (int s0 = at.blk * 256; s0 < a.nseq; s0 += a.blocks * 256) {
        const int s = s0 + t, lo = s < a.nseq ? min(max(off[s], 0), a.R) : 0, hi = s < a.nseq ? min(max(off[s + 1], 0), a.R) : 1;
        uint64_t m = __ballot(lo >= hi);
        for (; m; m &= m - 1) {
          const int64_t p = la_state_at<T, D>(a, at.b, s0 + wv.wave * 64 + __builtin_ctzll(m), hk);
          for (int i = lane; i < a.d * a.d; i += 64) J.S1[p + i] = J.S0 ? J.S0[p + i] : 0.f;
        }
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
  const T* pb = pk_at<T>(J.B, J.bs, at.b, hk * G);
  const T* pc = pk_at<T>(J.C, J.cs, at.b, hk * G);
  T* po = pk_at<T>(J.O, J.os, at.b, at.h);

  for (int tile = first; tile <= last; ++tile) {
    const int m0 = (rev ? a.tiles - 1 - tile : tile) * LA_T, rows = a.R - m0;
    // the sequences of this tile's rows
    __syncthreads();                                             // the last tile has been read
    if ((tile - first) % (LA_SPAN / LA_T) == 0) {
      const int t0 = rev ? m0 + LA_T - LA_SPAN : m0;
      lr.pr.template scan<256>(off, a.nseq, a.R, t0);
      if (t == 0) lr.t0 = t0;
      __syncthreads();
    }
    auto fetch = [&](int h) {
      if (h == 0) Stage::fetch(la, pa + (int64_t)m0 * J.as.r, J.as.r, rows, a.d, rev);
      Stage::fetch(lb, pb + h * J.bs.h + (int64_t)m0 * J.bs.r, J.bs.r, rows, a.d, rev);
      Stage::fetch(lc, pc + h * J.cs.h + (int64_t)m0 * J.cs.r, J.cs.r, rows, a.d, rev);
    };
    if constexpr (!PIECES) fetch(0);
    if (t < LA_T) {
      const int r = rev ? m0 + LA_T - 1 - t : m0 + t;
      int start, end;
      const bool in = r < a.R && lr.pr.range(lr.t0, r - lr.t0, start, end);
      const int rel = !in ? LA_NONE : max(rev ? m0 + LA_T - end : start - m0, -1);
      lr.rel[t] = rel;
      if constexpr (PIECES) {
        lr.seqend[t] = in && (rev ? r == start : r == end - 1);
      } else {                                                   // rows that go on into the next tile, rows that came from the one before
        wt[t] = t >= __builtin_amdgcn_readlane(rel, LA_T - 1) ? pw[LA_T - 1 - t] : 0.f;
        fac[t] = rel == -1 ? pw[t + 1] : 0.f;
      }
    }
    if (VEC && !PIECES) pk_landed();
    __syncthreads();
    const int mine = lr.rel[lane];
    if (tile == first && tile > 0 && __builtin_amdgcn_readlane(mine, 0) == -1) {      // what the first row's sequence brings from the blocks before
      int start, end;
      const int r = rev ? m0 + LA_T - 1 : m0;
      lr.pr.range(lr.t0, r - lr.t0, start, end);
      const int begin = rev ? a.tiles * LA_T - end : start;
      float* sum = a.sums + (((int64_t)at.job * a.B + at.b) * a.Hkv + hk) * a.blocks * (D * D);
      const float m1 = la_powm1(ld, a.per * LA_T);
#pragma unroll 1
      for (int k = a.scanned ? at.blk - 1 : begin / (a.per * LA_T); k < at.blk; ++k) {
        la_fade(s, m1);
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 v = *la_sum<D>(sum + (int64_t)k * (D * D), wv.cs, n, q, lane);
            s[n][4 * q] += v.x;
            s[n][4 * q + 1] += v.y;
            s[n][4 * q + 2] += v.z;
            s[n][4 * q + 3] += v.w;
          }
      }
    }
    const uint64_t there = __ballot(mine != LA_NONE);
    if (!there) continue;
    for (int p0 = PIECES ? __builtin_ctzll(there) : 0, p1; p0 < LA_T;) {
      const int val = __builtin_amdgcn_readlane(mine, PIECES ? p0 : LA_T - 1);
      const bool begins = PIECES && val >= 0;
      p1 = LA_T;
      if constexpr (PIECES) {
        const uint64_t m = __ballot(mine != val && lane > p0);
        if (m) p1 = __builtin_ctzll(m);
      }
      // rows of the state's update, and whether it comes late: against the order, what comes in behind the last row has not faded there
      const int c0 = PIECES ? p0 : val == LA_NONE ? LA_T : max(val, 0), late = begins && J.S0 && rev ? 1 : 0;
      if constexpr (PIECES) {
        if (begins) {
#pragma unroll
          for (int n = 0; n < D / 32; ++n) s[n] = pk_f16{};
          if (J.S0) la_load_state<T, D>(s, J, a, at.b, la_sequence(off, a.nseq, rev ? m0 + LA_T - 1 - p0 : m0 + p0), hk, wv);
        }
      }
      const bool brings = PIECES ? !begins || J.S0 : __builtin_amdgcn_readlane(mine, 0) == -1;
      const bool ends = keeps && lr.seqend[p1 - 1], updates = PIECES ? ends || (p1 == LA_T && tile < last) : c0 < LA_T && tile < last;
      pk_f16 acc[NTB];
#pragma unroll
      for (int n = 0; n < NTB; ++n) acc[n] = pk_f16{};
      for (int h = 0; h < G; ++h) {
        if (PIECES || h > 0) {
          __syncthreads();                                       // what the last pass reads has been read
          if (PIECES && t < LA_T) {
            wt[t] = t >= c0 && t < p1 ? pw[p1 - 1 - t] : 0.f;
            fac[t] = t >= p0 && t < p1 ? pw[t - p0 + 1 - late] : 0.f;
          }
          fetch(h);
          la_land<VEC>();
        }
        // a lane's piece of row l%32 of a tile is 16 (l/32) bytes on; addresses are formed where they are needed, or they would fill the registers
        uint32_t ar = (uint32_t)((lane & 31) * ROW + ((g ^ Tile::key(lane & 31)) << 4));
        asm volatile("" : "+v"(ar));
        if (forms) {                                             // (A B^T) . D
          pk_f16 y = pk_f16{};
          const unsigned char *xa = ta + 32 * qt * ROW, *xb = tb + 32 * qs * ROW;
#pragma unroll
          for (int i = 0; i < PkRow<T, D>::N; ++i) {
            typename PkRow<T, D>::Piece x, b;
            x.u = *reinterpret_cast<const uint4*>(xa + (ar ^ (uint32_t)(i << 5)));
            b.u = *reinterpret_cast<const uint4*>(xb + (ar ^ (uint32_t)(i << 5)));
            if constexpr (BF) {
              y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v, x.v, y, 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_32x32x2f32(b.e[e], x.e[e], y, 0, 0, 0);
            }
          }
          const int rel = lr.rel[32 * qt + (lane & 31)] - 32 * qs - 4 * g, self = 32 * (qt - qs) + (lane & 31) - 4 * g;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = 8 * (i >> 2) + (i & 3);
            y[i] = r >= rel && r <= self ? y[i] * D0[i] : 0.f;
          }
          if constexpr (BF) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              LaFrag hi, lo;
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                const float x0 = y[8 * k + 2 * p], x1 = y[8 * k + 2 * p + 1];
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
                  make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
          }
        }
        if (sums && brings && h == 0) {                          // Lambda A S
          const unsigned char* xa = ta + 32 * tb0 * ROW;
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
                typename PkRow<T, D>::Piece x[NTB];
#pragma unroll
                for (int n = 0; n < NTB; ++n) x[n].u = *reinterpret_cast<const uint4*>(xa + (ar ^ (uint32_t)((2 * kb + k) << 5)) + n * 32 * ROW);
#pragma unroll
                for (int n = 0; n < NTB; ++n) acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi.v, x[n].v, acc[n], 0, 0, 0);
#pragma unroll
                for (int n = 0; n < NTB; ++n) acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo.v, x[n].v, acc[n], 0, 0, 0);
              }
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int n = 0; n < NTB; ++n) {
                  typename PkRow<T, D>::Piece x;
                  x.u = *reinterpret_cast<const uint4*>(xa + (ar ^ (uint32_t)((4 * kb + q) << 5)) + n * 32 * ROW);
#pragma unroll
                  for (int e = 0; e < 4; ++e) acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(s[kb][4 * q + e], x.e[e], acc[n], 0, 0, 0);
                }
            }
          }
#pragma unroll
          for (int n = 0; n < NTB; ++n) {
            const int row = 32 * (tb0 + n) + (lane & 31);
            const float f = fac[row];
            const bool sees = PIECES ? row >= p0 && row < p1 : lr.rel[row] == -1;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][i] = sees ? f * acc[n][i] : 0.f;
          }
        }
        __syncthreads();
        if (sums) {                                              // the masked products with c
          uint32_t ap = (uint32_t)PkTile<bf16_raw, 64>::at(lane & 31, g * 16);
          uint32_t af = (uint32_t)PkTile<float, 64>::at(lane & 31, g * 16);
          if constexpr (BF) {
            asm volatile("" : "+v"(ap));
            LaFrag c[4];
            uint32_t odd = 0;
            const uint32_t at_c = la_cols_at<D, false>(lane);
#pragma unroll
            for (int k = 0; k < 4; ++k) la_cols<D>(c[k], lc, at_c, 16 * k, 32 * wv.cs);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int p = 0; p < 4; ++p) odd |= la_odd(c[k].u[p]);
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
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int n = 0; n < NTB; ++n) {
                if (k >= 2 && tb0 + n == 0) continue;
                const unsigned char* p = P + (ap ^ (uint32_t)(k << 5)) + 32 * (tb0 + n) * 128;
                const pk_bf8 hi = *reinterpret_cast<const pk_bf8*>(p), lo = *reinterpret_cast<const pk_bf8*>(p + 8192);
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[k].v, hi, acc[n], 0, 0, 0);
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(c[k].v, lo, acc[n], 0, 0, 0);
              }
            if (__builtin_expect(marks, 0)) la_mark<T, D, NTB>(acc, tc, wv, tb0, lr.rel);
          } else {
            asm volatile("" : "+v"(af));
            // a column's values of the two halves' rows; row 8 q + 4 g + e
            uint32_t ac = (uint32_t)Tile::at(4 * g, (32 * wv.cs + (lane & 31)) * 4);
            asm volatile("" : "+v"(ac));
            auto value = [&](int row) { return *reinterpret_cast<const float*>(tc + (ac ^ (uint32_t)(Tile::key(row) << 4)) + row * ROW); };
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) z = fmaf(0.f, value(8 * (i >> 2) + (i & 3)), z);
            const bool marks = __any(z != z);
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float c = value(8 * q + e);
                if (__builtin_expect(marks, 0) && (__float_as_uint(c) & 0x7f800000u) == 0x7f800000u) c = 0.f;
#pragma unroll
                for (int n = 0; n < NTB; ++n) {
                  if (q >= 4 && tb0 + n == 0) continue;
                  const float w = *reinterpret_cast<const float*>(P + (af ^ (uint32_t)(q << 5)) + 32 * (tb0 + n) * 256 + e * 4);
                  acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(c, w, acc[n], 0, 0, 0);
                }
              }
            if (__builtin_expect(marks, 0)) la_mark<T, D, NTB>(acc, tc, wv, tb0, lr.rel);
          }
          if (h == G - 1) {
#pragma unroll
            for (int n = 0; n < NTB; ++n) {
              const int j = 32 * (tb0 + n) + (lane & 31);
              if (lr.rel[j] == LA_NONE || (PIECES && (j < p0 || j >= p1))) continue;
              const pk_f16 one[1] = {acc[n]};
              pk_store_row<T, 1, VEC>(po + (int64_t)(rev ? m0 + LA_T - 1 - j : m0 + j) * J.os.r, one, J.fo, wv.cs, a.d, g);
            }
          }
        }
        if (updates && sums) {
          if (h == 0) {
            if (!PIECES && val >= 0) {                           // a sequence that began in this tile
#pragma unroll
              for (int n = 0; n < D / 32; ++n) s[n] = pk_f16{};
            } else {
              la_fade(s, la_powm1(ld, p1 - c0 - late));
            }
          }
          la_update<T, D, 1>(s, lb, lc, wt, c0, p1, c0 > 0 || p1 < LA_T, PIECES && J.S1 != nullptr, wv, 0);
        }
      }
      if (ends && (TH == 1 || wv.th == 0))
        la_store_state<T, D>(s, J.S1 + la_state_at<T, D>(a, at.b, la_sequence(off, a.nseq, rev ? m0 + LA_T - p1 : m0 + p1 - 1), hk), a.d,
                             J.fi * (rev ? pw[1] : 1.f), wv);
      if (!PIECES) break;
      const uint64_t rest = p1 < LA_T ? there >> p1 << p1 : 0;
      p0 = rest ? __builtin_ctzll(rest) : LA_T;
    }
  }
}

template <typename T, int D> int launch(const LaArgs& a, const LaForm& f, hipStream_t st) {
  int64_t n = 0;
  bool pieces = false;
  for (int j = 0; j < a.jobs; ++j) {
    n += (int64_t)a.blocks * a.B * a.job[j].heads;
    pieces = pieces || a.job[j].S0 || a.job[j].S1;
  }
  const dim3 grid((unsigned)n), block(256);
  if (f.vec && pieces) hipLaunchKernelGGL((la_main_kernel<T, D, true, true>), grid, block, 0, st, a);
  else if (f.vec) hipLaunchKernelGGL((la_main_kernel<T, D, true, false>), grid, block, 0, st, a);
  else if (pieces) hipLaunchKernelGGL((la_main_kernel<T, D, false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((la_main_kernel<T, D, false, false>), grid, block, 0, st, a);
  return launch_status();
}

}  // namespace

int la_main(const LaArgs& a, const LaForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
