// Linear attention: the walk over the tiles of a block (linear_attention.h).
#include "linear_attention.h"

namespace hfta {
namespace {

// of the wavefront's columns of c: NaN into the rows that see a value of the tile which is not finite
template <typename T, int D> __device__ __forceinline__ void la_mark(la_f4 (&acc)[4], const unsigned char* tc, const LaWave<D>& wv, const signed char* rel) {
  int c0 = 16 * wv.cs + 4 * wv.g;
  asm volatile("" : "+v"(c0));                                   // (nothing of this is worth a register outside)
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int t = 16 * n + wv.l, begin = rel[t];
#pragma unroll 1
    for (int r = 0; r < LA_T; ++r) {
      const bool sees = r >= begin && r <= t;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = Elem<T>::load(reinterpret_cast<const T*>(tc + LaTile<T, D>::at(r, (c0 + i) * (int)sizeof(T)))), y = sees ? x : 0.f;
        acc[n][i] += y - y;                                      // NaN, or nothing
      }
    }
  }
}

// A row's weight in the state's update, and the state's weight in a row, for two steps in turn
struct LaStep { float wt[LA_T], fac[LA_T]; };

// The masked products (A B^T) . D of a tile: six blocks of 16 rows t by 32 rows s (the other two are all zeros), 16 bytes a lane as the second product
// takes them; bf16: values, and behind them what is left; fp32: columns s of 16 each
struct LaP {
  static constexpr int PART = 1024, REST = 6 * PART, BYTES = 12 * PART;
  static __device__ __forceinline__ constexpr int block(int t, int s) { return s == 0 ? t : t + 2; }
};

// A workgroup's tiles, one step each; with several heads of B and C a step for each of them, with PIECES (states come in or go out) a step for each
// sequence of a tile.  The next tile of A is on its way while one is computed, those of B and C when this one's have been read.  A result takes
// the place of its rows of A, from where it is stored in whole pieces.  (Two workgroups of 128 columns of bf16 fill the LDS.)
template <typename T, int D, bool VEC, bool PIECES>
__global__ __launch_bounds__(4 * D, (sizeof(T) == 4 || (PIECES && D == 128) ? 2 : D == 128 ? 4 : 3)) void la_main_kernel(LaArgs a) {
  typedef LaStage<T, D, VEC> Stage;
  typedef LaTile<T, D> Tile;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NT = LaWave<D>::NT, WAVES = LaWave<D>::WAVES, ROW = Tile::ROW;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[4 * Stage::BYTES], P[LaP::BYTES];
  __shared__ PackedRows<LA_SPAN> pr;
  __shared__ __attribute__((aligned(16))) LaStep steps[2];
  __shared__ signed char rels[LA_SPAN / LA_T][LA_T];             // where the rows' sequences begin, of a span's tiles
  __shared__ uint64_t finals[LA_SPAN / LA_T];                    // rows that are their sequence's last one in the order of the walk
  __shared__ float pw[LA_T + 1], fade[LA_T + 1], dw[2 * LA_T + 1];      // lambda^n, la_faded(n); behind LA_T places of nothing lambda^n fo
  const LaWave<D> wave;
  const int t = threadIdx.x;
  la_touch(a);
  const LaPlace at(a, false);
  if (at.none) return;
  const LaJob& J = a.job[at.job];
  const int rev = J.rev, hk = at.h / J.ga, G = J.gb;
  const int32_t* off = a.off + (int64_t)at.b * (a.nseq + 1);
  const int first = at.blk * a.per, last = min(first + a.per, a.tiles) - 1;
  const bool keeps = PIECES && J.S1 && at.h % J.ga == 0;
  const int64_t lda = J.as.r, ldb = J.bs.r, ldc = J.cs.r, ldo = J.os.r;
  const T* pa = pk_at<T>(J.A, J.as, at.b, at.h);
  const T* pb = pk_at<T>(J.B, J.bs, at.b, hk * G);
  const T* pc = pk_at<T>(J.C, J.cs, at.b, hk * G);
  T* po = pk_at<T>(J.O, J.os, at.b, at.h);
  auto row0 = [&](int tile) __attribute__((always_inline)) { return (rev ? a.tiles - 1 - tile : tile) * LA_T; };       // a tile's first row in memory
  Stage sa, sb, sc;
  sa.init(lda, a.d, rev);
  sb.init(ldb, a.d, rev);
  sc.init(ldc, a.d, rev);
  const la_lds l0 = (la_lds)tiles;
  auto fetch_a = [&](int tile, int x) __attribute__((always_inline)) { sa.fetch(l0 + x * Stage::BYTES, pa + row0(tile) * lda, lda, a.R - row0(tile), a.d, rev); };
  const la_lds lb = l0 + 2 * Stage::BYTES, lc = l0 + 3 * Stage::BYTES;
  const unsigned char *tb = tiles + 2 * Stage::BYTES, *tc = tiles + 3 * Stage::BYTES;
  auto fetch_bc = [&](int tile, int h, int back = 0) __attribute__((always_inline)) {        // back: two tiles before their places
    const int m0 = row0(tile);
    sb.fetch(lb - back, pb + h * J.bs.h + m0 * ldb, ldb, a.R - m0, a.d, rev);
    sc.fetch(lc - back, pc + h * J.cs.h + m0 * ldc, ldc, a.R - m0, a.d, rev);
  };
  const float raw = a.ld[(int64_t)at.b * a.Hkv + hk];
  const int32_t warm = off[min(t, a.nseq)];                      // (on their way while the tables are formed)
  fetch_a(first, 0);
  if (a.mode != LA_WALK) fetch_bc(first, 0);
  la_f4 s[D / 16];
#pragma unroll
  for (int n = 0; n < D / 16; ++n) s[n] = la_f4{0.f, 0.f, 0.f, 0.f};
  float* const sum = a.sums + (((int64_t)J.sum * a.B + at.b) * a.Hkv + hk) * a.blocks * (D * D);
  const bool scanned = a.mode == LA_SCANNED && first > 0;
  if (scanned) la_load_sum<T, D>(s, sum + (int64_t)(at.blk - 1) * (D * D), J.turned, wave);        // (before it is known whether a sequence goes on here)
  const float ld = la_decay(raw);
  if (t <= LA_T) {
    pw[t] = la_pow(ld, t);
    fade[t] = la_faded(ld, t);
    dw[LA_T + t] = J.fo * la_pow(ld, t);
  }
  if (t < LA_T) dw[t] = 0.f;
  asm volatile("" :: "v"(warm));

  if constexpr (PIECES) {
    if (keeps)                                                   // sequences without rows, by all wavefronts
      for (int s0 = at.blk * 64; s0 < a.nseq; s0 += a.blocks * 64) {
        const int s = s0 + wave.lane, lo = s < a.nseq ? min(max(off[s], 0), a.R) : 0, hi = s < a.nseq ? min(max(off[s + 1], 0), a.R) : 1;
        uint64_t m = __ballot(lo >= hi);
        for (; m; m &= m - 1) {
          const int64_t p = la_state_at<T, D>(a, at.b, s0 + __builtin_ctzll(m), hk);
#pragma unroll 8
          for (int i = t; i < a.d * a.d; i += NT) J.S1[p + i] = J.S0 ? J.S0[p + i] : 0.f;
        }
      }
  }

  LaSpan span;
  auto look = [&](int tile) __attribute__((always_inline)) {     // up the sequences of the rows of this tile and the next ones
    const int t0 = rev ? row0(tile) + LA_T - LA_SPAN : row0(tile);
    pr.template scan<NT>(off, a.nseq, a.R, t0);
    span.take(pr, t0, wave.lane);
    for (int k = wave.cs; k < LA_SPAN / LA_T && tile + k <= last; k += WAVES) {
      const int m0 = row0(tile + k), r = rev ? LA_T - 1 - wave.lane : wave.lane;
      int start, end;
      const bool in = span.range(m0, r, start, end) && m0 + r < a.R;
      rels[k][wave.lane] = (signed char)(!in ? LA_NONE : max(rev ? m0 + LA_T - end : start - m0, -1));
      if constexpr (PIECES) {
        const uint64_t f = __ballot(in && m0 + r == (rev ? start : end - 1));
        if (wave.lane == 0) finals[k] = f;
      }
    }
    __syncthreads();
  };
  look(first);                                                   // (its barriers make the tables visible too)

  // what the first row's sequence brings from the blocks before
  if (first > 0) {
    int start, end;
    const int m0 = row0(first), r = rev ? LA_T - 1 : 0;
    const bool in = m0 + r < a.R && span.range(m0, r, start, end);
    const int begin = in ? rev ? a.tiles * LA_T - end : start : first * LA_T;
    if (begin >= first * LA_T) {
#pragma unroll
      for (int n = 0; n < D / 16; ++n) s[n] = la_f4{0.f, 0.f, 0.f, 0.f};
    } else if (a.mode == LA_SUMS) {
      const float f = la_faded(ld, a.per * LA_T);
#pragma unroll 1
      for (int k = begin / (a.per * LA_T); k < at.blk; ++k) {
        la_f4 v[D / 16];
        la_load_sum<T, D>(v, sum + (int64_t)k * (D * D), J.turned, wave);
        la_fade(s, f);
#pragma unroll
        for (int n = 0; n < D / 16; ++n) s[n] += v[n];
      }
    } else if (a.mode == LA_WALK) {
      // sequences are short: their rows up to here once more.  b's and c's tiles lie where the walk's will, and in the places of A's in turn
      if (PIECES && J.S0) la_load_state<T, D>(s, J, a, at.b, la_sequence(off, a.nseq, m0 + r), hk, wave);
      int tile = begin / LA_T, h = 0, i = 0;
      bool more;
      fetch_bc(tile, 0);
#pragma unroll 1
      do {
        const int c0 = max(begin - tile * LA_T, 0), n = LA_T - c0 - (PIECES && J.S0 && rev && tile == begin / LA_T ? 1 : 0), back = (i & 1) * 2 * Stage::BYTES;
        if (h == 0) la_fade(s, fade[n]);
        if (t < LA_T) steps[i & 1].wt[t] = t >= c0 ? pw[LA_T - 1 - t] : 0.f;
        la_land<VEC>();
        if (++h == G) {
          h = 0;
          ++tile;
        }
        more = tile < first;
        if (more) fetch_bc(tile, h, 2 * Stage::BYTES - back);
        if (c0 > 0) {
          la_clear<T, D>(lb - back, c0);
          __syncthreads();
        }
        la_update<T, D, false, PIECES>(s, lb - back, lc - back, steps[i & 1].wt, 0, LA_T, wave);
        ++i;
      } while (more);
      __syncthreads();
      if (i > 1) fetch_a(first, 0);
    }
  }
  if (a.mode == LA_WALK) fetch_bc(first, 0);

  int step = 0, x = 0;                                           // steps, and the place of this one's tile of A
  for (int tile = first; tile <= last; ++tile, x ^= 1) {
    const int m0 = row0(tile), in_span = (tile - first) % (LA_SPAN / LA_T);
    if (tile > first && in_span == 0) look(tile);                // (behind a barrier, at the end of the last tile)
    const signed char* rel = rels[in_span];
    LaWave<D> wv = wave.again();
    const int mine = rel[wv.lane];
    const uint64_t there = __ballot(mine != LA_NONE);
    const bool mixed = __any(mine > 0);                          // rows of several sequences, or of none
    // sequence by sequence, or all rows at once (also of a tile that has none: its successor's tiles are fetched)
    for (int p0 = PIECES && there ? __builtin_ctzll(there) : 0, p1; p0 < LA_T;) {
      const int val = __builtin_amdgcn_readlane(mine, PIECES ? p0 : LA_T - 1);
      const bool begins = PIECES && val >= 0 && val != LA_NONE;
      p1 = LA_T;
      if constexpr (PIECES) {
        const uint64_t m = __ballot(mine != val && wv.lane > p0);
        if (m) p1 = __builtin_ctzll(m);
      }
      const uint64_t rest = PIECES && p1 < LA_T ? there >> p1 << p1 : 0;
      // rows of the state's update, and whether it comes late: against the order, what comes in behind the last row has not faded there
      const int c0 = val == LA_NONE ? LA_T : PIECES ? p0 : max(val, 0), late = begins && J.S0 && rev ? 1 : 0;
      const bool ends = keeps && (finals[in_span] >> (p1 - 1) & 1);
      int seq = 0;
      if constexpr (PIECES) {
        if ((begins && J.S0) || ends) seq = la_sequence(off, a.nseq, m0 + (rev ? LA_T - 1 - p0 : p0));
        if (begins) {
#pragma unroll
          for (int n = 0; n < D / 16; ++n) s[n] = la_f4{0.f, 0.f, 0.f, 0.f};
          if (J.S0) la_load_state<T, D>(s, J, a, at.b, seq, hk, wave.again());
        }
      }
      const bool brings = PIECES ? !begins || J.S0 : __builtin_amdgcn_readlane(mine, 0) == -1;
      const bool updates = c0 < LA_T && (PIECES ? ends || (p1 == LA_T && tile < last) : tile < last);
      la_f4 acc[4];                                              // rows t = 16 n + l, columns 16 cs + 4 g + i
#pragma unroll
      for (int n = 0; n < 4; ++n) acc[n] = la_f4{0.f, 0.f, 0.f, 0.f};
      for (int h = 0; h < G; ++h, ++step) {
        LaStep& S = steps[step & 1];
        wv = wave.again();
        if (wv.cs == 0) {
          const int t = wv.lane;
          S.wt[t] = t >= c0 && t < p1 ? pw[p1 - 1 - t] : 0.f;
          S.fac[t] = PIECES ? (t >= p0 && t < p1 ? dw[LA_T + t - p0 + 1 - late] : 0.f) : mine == -1 ? dw[LA_T + t + 1] : 0.f;
        }
        const bool same = PIECES && G == 1 && (there & ((1ull << p0) - 1));       // the tiles, and the products of A and B, of the last step
        if (same) __syncthreads();
        else la_land<VEC>();
        const bool more_h = h + 1 < G, again = rest && G > 1, more_t = !rest && tile < last;       // the next step's tiles
        if (!more_h && more_t) fetch_a(tile + 1, x ^ 1);
        const unsigned char* ta = tiles + x * Stage::BYTES;
        // a lane's piece of row l of a tile is 16 g bytes on; addresses are formed where they are needed, or they would fill the registers
        wv = wave.again();
        const uint32_t ar = (uint32_t)Tile::at(wv.l, 16 * wv.g);
        if (there && !same) {
#pragma unroll
          for (int u = 0; u < 6; u += WAVES) {                   // (A B^T) . D: 16 rows t by 32 rows s
            if (u + wv.cs >= 6) break;
            // blocks 0 and 4 are half the others' work (their rows see the first sixteen of s only): four wavefronts take 0 and 5, 1 and 4, 2, 3
            const int unit = WAVES == 4 && u > 0 ? 5 - wv.cs : u + wv.cs, ti = unit < 4 ? unit : unit - 2, si = unit < 4 ? 0 : 1;
            const bool half = unit == 0 || unit == 4;
            la_f4 y[2] = {la_f4{0.f, 0.f, 0.f, 0.f}, la_f4{0.f, 0.f, 0.f, 0.f}};
            const unsigned char *xr = ta + 16 * ti * ROW, *br = tb + 32 * si * ROW;
#pragma unroll
            for (int i = 0; i < ROW / 64; ++i) {
              union { uint4 u; pk_bf8 v; float e[4]; } q, b[2];
              q.u = *reinterpret_cast<const uint4*>(xr + (ar ^ (uint32_t)(i << 6)));
#pragma unroll
              for (int k = 0; k < 2; ++k) b[k].u = *reinterpret_cast<const uint4*>(br + (ar ^ (uint32_t)(i << 6)) + 16 * k * ROW);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                if (k == 1 && half) break;
                if constexpr (BF) {
                  y[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[k].v, q.v, y[k], 0, 0, 0);
                } else {
#pragma unroll
                  for (int e = 0; e < 4; ++e) y[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[k].e[e], q.e[e], y[k], 0, 0, 0);
                }
              }
            }
            const LaWave<D> wu = wave.again();
            const int self = 16 * ti + wu.l - 32 * si - 4 * wu.g;       // s counts from 32 si + 4 g: 16 k + i
            if (mixed) {
              const int from = rel[16 * ti + wu.l] - 32 * si - 4 * wu.g;
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[k][i] = 16 * k + i >= from ? y[k][i] : 0.f;
            }
            const float* decay = dw + (LA_T - 19 + self);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int i = 0; i < 4; ++i) y[k][i] = 16 * k + i <= self ? y[k][i] * decay[19 - 16 * k - i] : 0.f;
            unsigned char* to = P + unit * LaP::PART + wu.lane * 16;
            if constexpr (BF) {
              LaFrag hi, lo;
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                float x0 = y[p >> 1][2 * (p & 1)], x1 = y[p >> 1][2 * (p & 1) + 1];
                hi.u[p] = la_word(x0, x1);
                lo.u[p] = pack_bf16x2(x0, x1);
              }
              *reinterpret_cast<uint4*>(to) = make_uint4(hi.u[0], hi.u[1], hi.u[2], hi.u[3]);
              *reinterpret_cast<uint4*>(to + LaP::REST) = make_uint4(lo.u[0], lo.u[1], lo.u[2], lo.u[3]);
            } else {
#pragma unroll
              for (int k = 0; k < 2; ++k) *reinterpret_cast<la_f4*>(to + k * LaP::REST) = y[k];
            }
          }
        }
        if (brings && h == 0) {                                  // Lambda A S
          const uint32_t as = (uint32_t)Tile::at(wv.l, 8 * wv.g);
#pragma unroll
          for (int j = 0; j < ROW / 64; ++j) {
            union { uint4 u; uint2 h[2]; pk_bf8 v; float e[4]; } q[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              if constexpr (BF) {                                // columns 32 j + 4 g + 0..3 and 16 on, as the state's rows lie
#pragma unroll
                for (int k = 0; k < 2; ++k) q[n].h[k] = *reinterpret_cast<const uint2*>(ta + (as ^ (uint32_t)(j << 6 | k << 5)) + 16 * n * ROW);
              } else {
                q[n].u = *reinterpret_cast<const uint4*>(ta + (ar ^ (uint32_t)(j << 6)) + 16 * n * ROW);
              }
            }
            if constexpr (BF) {
              LaFrag hi, lo;
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                float x0 = s[2 * j + (p >> 1)][2 * (p & 1)], x1 = s[2 * j + (p >> 1)][2 * (p & 1) + 1];
                hi.u[p] = la_word(x0, x1);
                lo.u[p] = pack_bf16x2(x0, x1);
              }
#pragma unroll
              for (int n = 0; n < 4; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi.v, q[n].v, acc[n], 0, 0, 0);
#pragma unroll
              for (int n = 0; n < 4; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo.v, q[n].v, acc[n], 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(s[j][e], q[n].e[e], acc[n], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);                   // (here and below: no more reads of LDS in flight than there are registers for)
          }
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const int row = 16 * n + wv.l;
            acc[n] *= S.fac[row];
            if (PIECES || mixed) {
              const bool sees = PIECES ? row >= p0 && row < p1 : rel[row] == -1;
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[n][i] = sees ? acc[n][i] : 0.f;
            }
          }
        }
        __syncthreads();
        if (there) {                                             // the masked products with c
          wv = wave.again();
          const unsigned char* pl = P + wv.lane * 16;
          if constexpr (BF) {
            LaFrag c[2];
            uint32_t odd = 0;
            const uint32_t at_c = la_cols_at<D>(wv.lane);
#pragma unroll
            for (int k = 0; k < 2; ++k) la_cols<D>(c[k], lc, at_c, 32 * k, 16 * wv.cs);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int p = 0; p < 4; ++p) odd |= la_odd(c[k].u[p]);
            const bool marks = __any(odd & 0x80008000u);
            if (__builtin_expect(marks, 0)) {
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                  const uint32_t o = la_odd(c[k].u[p]);
                  c[k].u[p] &= (o & 0x8000u ? 0u : 0xffffu) | (o & 0x80000000u ? 0u : 0xffff0000u);
                }
            }
#pragma unroll
            for (int u0 = 0; u0 < 6; u0 += 2) {                  // blocks (0, 0) (1, 0), (2, 0) (3, 0), (2, 1) (3, 1)
              const int n0 = u0 < 4 ? u0 : 2, k = u0 < 4 ? 0 : 1;
              pk_bf8 hi[2], lo[2];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                hi[i] = *reinterpret_cast<const pk_bf8*>(pl + (u0 + i) * LaP::PART);
                lo[i] = *reinterpret_cast<const pk_bf8*>(pl + (u0 + i) * LaP::PART + LaP::REST);
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) acc[n0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c[k].v, hi[i], acc[n0 + i], 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 2; ++i) acc[n0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c[k].v, lo[i], acc[n0 + i], 0, 0, 0);
            }
            if (__builtin_expect(marks, 0)) la_mark<T, D>(acc, tc, wv, rel);
          } else {
            // a column's values of the four quarters' rows 16 q + 4 g + e
            const uint32_t ac = (uint32_t)Tile::at(4 * wv.g, (16 * wv.cs + wv.l) * 4);
            auto value = [&](int row) __attribute__((always_inline)) { return *reinterpret_cast<const float*>(tc + (ac ^ (uint32_t)(Tile::key(row) << 4)) + row * ROW); };
            float c[16], z = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              c[i] = value(16 * (i >> 2) + (i & 3));
              z = fmaf(0.f, c[i], z);
            }
            const bool marks = __any(z != z);
            if (__builtin_expect(marks, 0)) {
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if ((__float_as_uint(c[i]) & 0x7f800000u) == 0x7f800000u) c[i] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int n = 0; n < 4; ++n) {
                if (n < q) continue;                             // (sixteen rows s behind these)
                const la_f4 w = *reinterpret_cast<const la_f4*>(pl + LaP::block(n, q >> 1) * LaP::PART + (q & 1) * LaP::REST);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(c[4 * q + e], w[e], acc[n], 0, 0, 0);
              }
            if (__builtin_expect(marks, 0)) la_mark<T, D>(acc, tc, wv, rel);
          }
          if (h == G - 1) {                                      // the result's rows in place of A's
            wv = wave.again();
            const uint32_t ao = (uint32_t)Tile::at(wv.l, (16 * wv.cs + 4 * wv.g) * (int)sizeof(T));
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const int row = 16 * n + wv.l;
              if (PIECES && (row < p0 || row >= p1)) continue;
              unsigned char* p = tiles + x * Stage::BYTES + ao + 16 * n * ROW;
              const la_f4 o = acc[n];
              if constexpr (BF) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
              else *reinterpret_cast<la_f4*>(p) = o;
            }
          }
        }
        if (updates) {
          wv = wave.again();
          if (h == 0) {
            if (!PIECES && val >= 0) {                           // a sequence that began in this tile
#pragma unroll
              for (int n = 0; n < D / 16; ++n) s[n] = la_f4{0.f, 0.f, 0.f, 0.f};
            } else {
              la_fade(s, fade[p1 - c0 - late]);
            }
          }
          if (PIECES && (c0 > 0 || p1 < LA_T)) {
            la_update<T, D, true, PIECES>(s, lb, lc, S.wt, c0, p1, wv);
          } else {
            if (c0 > 0) {                                        // rows of other sequences: what stands there does not matter
              __syncthreads();
              la_clear<T, D>(lb, c0);
              __syncthreads();
            }
            la_update<T, D, false, PIECES>(s, lb, lc, S.wt, 0, LA_T, wv);
          }
        }
        __syncthreads();                                         // the step's tiles have been read, its results lie in LDS
        if (more_h || again) fetch_bc(tile, more_h ? h + 1 : 0);
        else if (more_t) fetch_bc(tile + 1, 0);
      }
      if (ends) la_store_state<T, D>(s, J.S1 + la_state_at<T, D>(a, at.b, seq, hk), a.d, J.fi * (rev ? pw[1] : 1.f), wave.again());
      if (!PIECES) break;
      p0 = rest ? __builtin_ctzll(rest) : LA_T;
    }
    // the tile's results, as its rows of A came in
    if (there) {
      const unsigned char* from = tiles + x * Stage::BYTES;
      wv = wave.again();
#pragma unroll
      for (int n = 0; n < Stage::N; ++n) {
        const int q = n * NT + wv.t(), row = q / Tile::PPR, c = ((q % Tile::PPR) ^ Tile::key(row)) * Stage::EPP;
        if (rel[row] == LA_NONE || c >= a.d) continue;
        union { uint4 u; piece_u4 p; T e[Stage::EPP]; } v;
        v.u = *reinterpret_cast<const uint4*>(from + q * 16);
        T* p = po + (int64_t)(m0 + (rev ? LA_T - 1 - row : row)) * ldo + c;
        if constexpr (VEC) {
          *reinterpret_cast<uint4*>(p) = v.u;
        } else if (c + Stage::EPP <= a.d) {
          *reinterpret_cast<piece_u4*>(p) = v.p;
        } else {
          for (int e = 0; e < Stage::EPP; ++e)
            if (c + e < a.d) p[e] = v.e[e];
        }
      }
    }
  }
}

template <typename T, int D> int launch(const LaArgs& a, const LaForm& f, hipStream_t st) {
  const dim3 grid((unsigned)LaPlace::count(a, false)), block(LaWave<D>::NT);
  if (f.vec && f.pieces) hipLaunchKernelGGL((la_main_kernel<T, D, true, true>), grid, block, 0, st, a);
  else if (f.vec) hipLaunchKernelGGL((la_main_kernel<T, D, true, false>), grid, block, 0, st, a);
  else if (f.pieces) hipLaunchKernelGGL((la_main_kernel<T, D, false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((la_main_kernel<T, D, false, false>), grid, block, 0, st, a);
  return launch_status();
}

}  // namespace

int la_main(const LaArgs& a, const LaForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
