// Linear attention with a decay for each key head over packed sequences, forward and backward (fusion rules table row
// "MultiheadAttention": the projections are fused Linears, this is what stands between them).
//
//   S_t = lambda S_t-1 + k_t v_t^T,   ctx_t = scale q_t S_t            lambda = exp(log_decay), S in front of a sequence: state_in, or zeros
//
// All four results are sums of one form, f(A, B, C)_t = sum_{s <= t} lambda^(t-s) (a_t . b_s) c_s, over rows in order or against it:
//   ctx = scale f(q, k, v);   dq = scale f(dctx, v, k);   against the order: dv = scale f(k, q, dctx), dk = scale f(v, dctx, q), heads of a group added
//
// Tile by tile of 64 rows, with the state S of the rows before (b's columns by c's columns):
//   O = ((A B^T) . D) C + Lambda A S,   S <- lambda^64 S + (W B)^T C        D_ts = lambda^(t-s), s <= t;  W_ss = lambda^(63-s)
// so that a row costs 2 (64 + 64 + 2 d) d products instead of a walk through a d x d state.
//
// Tiles are stretches of the packed rows, whatever sequences they hold: D sees rows of one sequence, Lambda rows of the one that came
// from the tile before, W rows of the one that goes on into the next.  Against the order everything is mirrored: row j of a tile is its
// row 63 - j in memory.  Blocks of tiles run side by side: a first launch forms the state that each block's last sequence
// takes with it, a second adds them up along each sequence, or, where blocks are few, the third does that for itself before it walks its tiles.
//
// A wavefront keeps 32 columns of c of the state in the matrix instruction's accumulators, fp32, for the whole walk; they are
// the operand of the product with A without a shuffle, because the update gives b's columns to the accumulator's rows in the order in which
// rows of A lie in registers.  (A B^T) . D passes through LDS.  bf16: what is rounded to bf16 as an operand (S, W C, the masked
// products) goes in as two words, value and rest, and W C as three where states are returned: results have the error of their own rounding alone.
//
// Entries that a row does not see are taken out by selects; values of C that are not finite and lie in a tile beside rows that do
// not see them are taken out of the product and put back as NaN into the rows that do.
#pragma once
#include "attention_packed.h"
#include "pieces.h"

namespace hfta {

constexpr int LA_T = 64;                                         // rows of a tile
constexpr int LA_SPAN = 512;                                     // rows whose sequences are looked up at once

typedef __attribute__((address_space(3))) unsigned char* la_lds;

struct LaJob {
  const void *A, *B, *C;
  void* O;
  PkStr as, bs, cs, os;
  const float* S0;                 // states in front of the first row (NULL: zeros), and behind the last (NULL: not wanted)
  float* S1;
  int rev;                         // against the order
  int flip;                        // the state's rows and columns change places in memory
  int heads, ga, gb;               // workgroups' heads of a model; heads of A (B and C) that belong to one of them: h / ga, h * gb ..
  float fo, fi;                    // results times fo, states in memory times 1 / fi
};
struct LaArgs {
  LaJob job[3];
  const int32_t* off;
  const float* ld;
  float* sums;                     // [job][model][key head][block][D * D], as accumulators lie
  int* spans;                      // [job][model][block]: 0: no sequence goes on behind the block, 1: one that began in it, 2: one from before it
  int B, R, nseq, Hkv, d, jobs, tiles, per, blocks;              // tiles in all and of a block, blocks
  int scanned;                     // sums are added up along the sequences already
};
struct LaForm { bool bf16, vec; };
int la_states(const LaArgs& a, const LaForm& f, hipStream_t st); // linear_attention_states.hip
int la_main(const LaArgs& a, const LaForm& f, hipStream_t st);   // linear_attention_main.hip
static inline int la_pad(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

// lambda^n and lambda^n - 1 with the argument's rounding made good; n = 0: 1 and 0 whatever lambda
__device__ __forceinline__ float la_decay(float ld) { return ld > 0.f ? 0.f : ld; }      // (a NaN stays one)
__device__ __forceinline__ float la_pow(float g, int n) {
  const float x = (float)n * g, e = fmaf((float)n, g, -x), y = expf(x);
  return n == 0 ? 1.f : x < -100.f ? 0.f : fmaf(y, e, y);
}
__device__ __forceinline__ float la_powm1(float g, int n) { return n == 0 ? 0.f : expm1f((float)n * g); }

// A wavefront's role: column block of c, block of 32 rows where two wavefronts share the columns
template <int D> struct LaWave {
  static constexpr int CS = D / 32, TH = 4 / CS, NTB = TH == 1 ? 2 : 1;
  int lane, wave, g, cs, th;
  __device__ __forceinline__ LaWave() {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    g = lane >> 5;
    cs = wave % CS;
    th = wave / CS;
  }
};

// 64 rows of a [row][D] matrix into LDS, rows that are not there and columns from d on zero; FLIP: the last row first
template <typename T, int D, bool VEC> struct LaStage {
  typedef PkTile<T, D> Tile;
  static constexpr int BYTES = LA_T * Tile::ROW, PIECES = BYTES / 16, N = PIECES / 256, EPP = 16 / (int)sizeof(T);
  static_assert(PIECES % 256 == 0, "whole pieces for every thread");
  // src: the tile's first row in memory, rows: how many there are
  static __device__ __forceinline__ void fetch(la_lds tile, const T* src, int64_t ld, int rows, int d, bool flip) {
    rows = min(rows, LA_T);
    if constexpr (VEC) {
      const uint32_t bytes = rows > 0 ? (uint32_t)((rows - 1) * (int)ld + d) * (uint32_t)sizeof(T) : 0u;
      const dma_i32x4 rs = dma_rsrc(src, bytes);
      const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)tile);
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int q = n * 256 + (int)threadIdx.x, row = q / Tile::PPR, byte = ((q % Tile::PPR) ^ Tile::key(row)) * 16, at = flip ? LA_T - 1 - row : row;
        const uint32_t off = byte < d * (int)sizeof(T) ? (uint32_t)(at * (int)ld) * (uint32_t)sizeof(T) + (uint32_t)byte : PK_OUT;
        dma_load(lds + (uint32_t)(n * 256 + wave * 64) * 16u, off, rs);
      }
    } else {
      union { piece_u4 u; T e[EPP]; } v;
#pragma unroll 1
      for (int n = 0; n < N; ++n) {
        const int q = n * 256 + (int)threadIdx.x, row = q / Tile::PPR, byte = ((q % Tile::PPR) ^ Tile::key(row)) * 16, at = flip ? LA_T - 1 - row : row;
        const int c = byte / (int)sizeof(T);
        const T* p = src + (int64_t)at * ld + c;
        v.u = piece_u4{0, 0, 0, 0};
        if (at < rows) {
          if (c + EPP <= d) v.u = *reinterpret_cast<const piece_u4*>(p);
          else
            for (int e = 0; e < EPP; ++e)
              if (c + e < d) v.e[e] = p[e];
        }
        *(__attribute__((address_space(3))) piece_u4*)(tile + q * 16) = v.u;
      }
    }
  }
};
// until the loads into LDS have landed, for all wavefronts
template <bool VEC> __device__ __forceinline__ void la_land() {
  if constexpr (VEC) pk_landed();
  __syncthreads();
}

// The rows of a tile: where each one's sequence begins, counted in the tile's rows in the order of the walk; -1: before it, LA_NONE: in none
constexpr int LA_NONE = 1 << 20;
struct LaRows {
  PackedRows<LA_SPAN> pr;
  int t0;                          // (of the span, in memory)
  int rel[LA_T];
  int seqend[LA_T];                // whether the row is its sequence's last one in the order of the walk
};

// bf16 pairs with infinities and NaNs have bit 15 of a half set in the result
__device__ __forceinline__ uint32_t la_odd(uint32_t u) { return (u & 0x7f807f80u) + 0x00800080u; }

typedef __attribute__((address_space(3))) pk_s4* la_lds4;
union LaFrag { uint32_t u[4]; pk_s4 h[2]; pk_bf8 v; bf16_raw e[8]; };

// Columns of a staged bf16 tile over 16 rows as a matrix operand: lane l holds column col0 + l%32 (SWAP: with bits 2 and 3 of l exchanged), its
// slots rows row0 + 4 (l/32) + 0..3 and 8 + 4 (l/32) + 0..3.  row0: a multiple of 16, col0: of 32
template <int D, bool SWAP> __device__ __forceinline__ uint32_t la_cols_at(int lane) {
  const int r = lane & 15, q = SWAP ? ((r & 1) << 1 | (r >> 1 & 1)) : r & 3;
  uint32_t a = (uint32_t)PkTile<bf16_raw, D>::at(4 * (lane >> 5) + (r >> 2), (16 * ((lane >> 4) & 1) + 4 * q) * 2);
  asm volatile("" : "+v"(a));                                    // (formed where it is needed)
  return a;
}
template <int D> __device__ __forceinline__ void la_cols(LaFrag& f, la_lds tile, uint32_t at, int row0, int col0) {
#pragma unroll
  for (int h = 0; h < 2; ++h)                                    // eight rows on: another bit of the key
    f.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((la_lds4)(tile + (at ^ (uint32_t)(col0 << 1 | h << 5)) + (row0 + 8 * h) * PkTile<bf16_raw, D>::ROW));
}

// A state in the accumulators of the wavefronts: s[kb], rows b's columns 32 kb + .., columns c's column 32 cs + lane % 32
template <typename T> __device__ __forceinline__ int la_row(int i, int g) {       // row of accumulator i, 0..31
  return sizeof(T) == 2 ? 16 * (i >> 3) + 8 * g + 4 * (i >> 2 & 1) + (i & 3) : 8 * (i >> 2) + 4 * g + (i & 3);
}
// its place in a block's sums
template <int D> __device__ __forceinline__ float4* la_sum(float* sums, int cs, int kb, int q, int lane) {
  return reinterpret_cast<float4*>(sums) + ((cs * (D / 32) + kb) * 4 + q) * 64 + lane;
}

// s += sum over tile rows [c0, c1) of w[row] b[row]^T c[row], w: LDS.  STEP: a wavefront takes every STEP-th sixteen rows from `from` on.
// `part`: rows outside of [c0, c1) may hold anything (else there are none).  three: c w as three words
template <typename T, int D, int STEP>
__device__ __forceinline__ void la_update(pk_f16 (&s)[D / 32], la_lds tb, la_lds tc, const float* w, int c0, int c1,
                                          bool part, bool three, const LaWave<D>& wv, int from) {
  const int lane = wv.lane, g = wv.g;
  if constexpr (sizeof(T) == 2) {
    const uint32_t at = la_cols_at<D, false>(lane), swapped = la_cols_at<D, true>(lane);
#pragma unroll
    for (int ks = 0; ks < LA_T / 16; ks += STEP) {
      const int row0 = 16 * (ks + from);
      LaFrag c, hi, lo, ll;
      la_cols<D>(c, tc, at, row0, 32 * wv.cs);
      const float4 w0 = *reinterpret_cast<const float4*>(w + row0 + 4 * g), w1 = *reinterpret_cast<const float4*>(w + row0 + 8 + 4 * g);
      const float wt[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
      uint32_t in = 0xffu;                                       // slots whose rows take part
      if (__builtin_expect(part, 0)) {
        in = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int row = row0 + 4 * g + (e & 3) + 8 * (e >> 2);
          if (row >= c0 && row < c1) in |= 1u << e;
        }
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float x0 = __uint_as_float(c.u[p] << 16) * wt[2 * p], x1 = __uint_as_float(c.u[p] & 0xffff0000u) * wt[2 * p + 1];
        if (__builtin_expect(part, 0)) {
          if (!(in >> (2 * p) & 1)) x0 = 0.f;
          if (!(in >> (2 * p + 1) & 1)) x1 = 0.f;
        }
        hi.u[p] = pack_bf16x2(x0, x1);
        x0 -= __uint_as_float(hi.u[p] << 16);
        x1 -= __uint_as_float(hi.u[p] & 0xffff0000u);
        lo.u[p] = pack_bf16x2(x0, x1);
        if (three) {
          x0 -= __uint_as_float(lo.u[p] << 16);
          x1 -= __uint_as_float(lo.u[p] & 0xffff0000u);
          ll.u[p] = pack_bf16x2(x0, x1);
        }
      }
#pragma unroll
      for (int kb = 0; kb < D / 32; ++kb) {
        LaFrag b;
        la_cols<D>(b, tb, swapped, row0, 32 * kb);
        if (__builtin_expect(part, 0)) {
#pragma unroll
          for (int p = 0; p < 4; ++p) b.u[p] &= (in >> (2 * p) & 1 ? 0xffffu : 0u) | (in >> (2 * p + 1) & 1 ? 0xffff0000u : 0u);
        }
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v, hi.v, s[kb], 0, 0, 0);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v, lo.v, s[kb], 0, 0, 0);
        if (three) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v, ll.v, s[kb], 0, 0, 0);
      }
    }
  } else {
    typedef PkTile<T, D> Tile;
    uint32_t at = (uint32_t)Tile::at(4 * g, (lane & 31) * 4);    // row 16 ks + 8 (i / 4) + 4 g + i % 4: other bits of the key, or none
    asm volatile("" : "+v"(at));
#pragma unroll 1
    for (int ks = from; ks < LA_T / 16; ks += STEP)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 8 * (i >> 2) + (i & 3), row = 16 * ks + r + 4 * g;
        const uint32_t to = (uint32_t)(16 * ks + r) * Tile::ROW, key = (uint32_t)Tile::key(r) << 4;
        float c = *(__attribute__((address_space(3))) const float*)(tc + (at ^ (key ^ (uint32_t)(wv.cs << 7))) + to) * w[row];
        const bool out = part && (row < c0 || row >= c1);
        if (out) c = 0.f;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
          float b = *(__attribute__((address_space(3))) const float*)(tb + (at ^ (key ^ (uint32_t)(kb << 7))) + to);
          if (out) b = 0.f;
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(b, c, s[kb], 0, 0, 0);
        }
      }
  }
}

// a sequence's state from and to memory
template <typename T, int D> __device__ __forceinline__ int64_t la_state_at(const LaArgs& a, int b, int seq, int hk) {
  return (((int64_t)b * a.nseq + seq) * a.Hkv + hk) * a.d * a.d;
}
template <typename T, int D>
__device__ __forceinline__ void la_load_state(pk_f16 (&s)[D / 32], const LaJob& J, const LaArgs& a, int b, int seq, int hk, const LaWave<D>& wv) {
  const float* p = J.S0 + la_state_at<T, D>(a, b, seq, hk);
  const int col = 32 * wv.cs + (wv.lane & 31), rs = J.flip ? 1 : a.d, cs = J.flip ? a.d : 1;
  const float f = 1.f / J.fi;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = 32 * n + la_row<T>(i, wv.g);
      s[n][i] = row < a.d && col < a.d ? f * p[row * rs + col * cs] : 0.f;
    }
}

template <int N> __device__ __forceinline__ void la_fade(pk_f16 (&s)[N], float m1) {       // s times 1 + m1
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[n][i] = fmaf(s[n][i], m1, s[n][i]);
}

// Workgroup -> (job, model, head of the job, block)
struct LaPlace {
  int job, b, h, blk;
  __device__ __forceinline__ LaPlace(const LaArgs& a, bool key_heads) {
    int64_t x = blockIdx.x;
    for (job = 0;; ++job) {
      const int64_t n = (int64_t)a.blocks * a.B * (key_heads ? a.Hkv : a.job[job].heads);
      if (x < n || job == a.jobs - 1) break;
      x -= n;
    }
    const int heads = key_heads ? a.Hkv : a.job[job].heads, bh = (int)(x % ((int64_t)a.B * heads));
    blk = (int)(x / ((int64_t)a.B * heads));
    b = bh / heads;
    h = bh % heads;
  }
};

}  // namespace hfta
