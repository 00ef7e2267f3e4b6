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
// row 63 - j in memory.  Blocks of tiles run side by side.  What a block's first row brings from the blocks before it comes, by a rule on sizes: from a
// first launch, which forms the state that each block's last sequence takes with it, added up by each block or, where there are many, along
// the sequences by a second launch; or, where sequences are short, from their rows in those blocks, walked once more.
//
// A wavefront keeps 16 columns of c of the state in the matrix instruction's accumulators, fp32, for the whole walk (D / 16 wavefronts are a
// workgroup); they are the operand of the product with A without a shuffle, because the update gives b's columns to the accumulator's rows in
// the order in which rows of A are read.  (A B^T) . D passes through LDS.  bf16: what is rounded to bf16 as an operand (S, W C, the masked
// products) goes in as two words, value and rest, and W C as three where states are returned: results have the error of their own rounding alone.
//
// Nothing bounds it alone.  2 x 16384 rows, 8 heads of 128 bf16, backward, 238 us: rows and results pass at 3.4 TB/s, LDS is active 37 % of the time, matrix
// instructions 21 %; 44 % of wavefront cycles wait for memory, LDS or a barrier and 26 % for an instruction to issue, along the chain
// products -> LDS -> products -> state of a tile.  Two workgroups of 128 columns or three of 64 on a compute unit fill each other's waits.
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
  int ga, gb;                      // a workgroup has a head h of A; the key head is h / ga, and it has gb heads of B and C
  float fo, fi;                    // results times fo, states in memory times 1 / fi
  int sum, turned;                 // which blocks' sums are its states, and whether they are of C and B instead (rows and columns change places)
};
enum { LA_ALONE = 0, LA_SUMS = 1, LA_SCANNED = 2, LA_WALK = 3 };   // one block; sums of blocks, added up by each block or along the sequences; none
struct LaArgs {
  LaJob job[3];                    // by sum first: job[i] forms sum i for i < nsums
  const int32_t* off;
  const float* ld;
  float* sums;                     // [sum][model][key head][block][D * D], as accumulators lie
  int* spans;                      // [sum][model][block]: 0: no sequence goes on behind the block, 1: one that began in it, 2: one from before it
  int B, R, nseq, Hkv, d, jobs, nsums, tiles, per, blocks;       // tiles in all and of a block, blocks
  int mode;
  PkDiv by_heads, by_hq, by_key_heads, by_hkv;                   // B times query heads, query heads, and of key heads
};
struct LaForm { bool bf16, vec, pieces; };                     // storage, rows in 16-byte pieces, states that come in or go out
int la_states(const LaArgs& a, const LaForm& f, hipStream_t st); // linear_attention_states.hip
int la_main(const LaArgs& a, const LaForm& f, hipStream_t st);   // linear_attention_main.hip
static inline int la_pad(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

// lambda^n with the argument's rounding made good; n = 0: 1 whatever lambda
__device__ __forceinline__ float la_decay(float ld) { return ld > 0.f ? 0.f : ld; }      // (a NaN stays one)
__device__ __forceinline__ float la_pow(float g, int n) {
  const float x = (float)n * g, e = fmaf((float)n, g, -x), y = expf(x);
  return n == 0 ? 1.f : x < -100.f ? 0.f : fmaf(y, e, y);
}
// What a state is multiplied by, in one number: lambda^n - 1 (at most 0) where at least half of the state is left, which a rounded lambda^n would
// make forget at another rate, the same way in every tile; lambda^n itself (above 0) where less is left, of which beside -1 only 2^-25 / lambda^n would be
// right.  Nothing left: -1.
__device__ __forceinline__ float la_faded(float g, int n) {
  const float y = la_pow(g, n);
  return y >= 0.5f ? n == 0 ? 0.f : expm1f((float)n * g) : y == 0.f ? -1.f : y;
}

// A staged tile: rows of D columns without padding, as the loads into LDS leave them; piece p (16 bytes) of row r lies at place p ^ key(r).  Sixteen
// rows' reads of one piece cover all 64 banks, and so do a transpose read's eight rows of two pieces and (fp32) four rows of four.
template <typename T, int D> struct LaTile {
  static constexpr int ROW = D * (int)sizeof(T), PPR = ROW / 16;
  static __device__ __forceinline__ constexpr int key(int r) {
    if (sizeof(T) == 2)
      return PPR == 16 ? (r & 3) << 2 | (r >> 2 & 1) << 1 | (r >> 3 & 1) : PPR == 8 ? (r >> 1 & 3) << 1 | (r >> 3 & 1) : (r >> 2 & 1) << 1 | (r >> 3 & 1);
    return PPR >= 16 ? (r >> 2 & 3) << 2 | (r & 3) : (r >> 2 & 1) << 2 | (r >> 3 & 1) << 1 | (r >> 1 & 1);
  }
  static __device__ __forceinline__ int at(int r, int byte) { return r * ROW + (((byte >> 4) ^ key(r)) << 4) + (byte & 15); }
};

typedef float la_f4 __attribute__((ext_vector_type(4)));
// A wavefront's role: it has columns 16 cs + l%16 of c; a lane's quarter g = l / 16
template <int D> struct LaWave {
  static constexpr int WAVES = D / 16, NT = 64 * WAVES, KT = D / 16;      // accumulators of a state: KT blocks of 16 x 16
  int lane, cs, l, g;
  __device__ __forceinline__ LaWave() {
    lane = threadIdx.x & 63;
    cs = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    l = lane & 15;
    g = lane >> 4;
  }
  // the same once more, hidden from the compiler: what follows from it is formed where it is needed, not kept in registers from before a loop
  __device__ __forceinline__ LaWave again() const {
    LaWave w = *this;
    asm volatile("" : "+v"(w.lane));
    w.l = w.lane & 15;
    w.g = w.lane >> 4;
    return w;
  }
  __device__ __forceinline__ int t() const { return 64 * cs + lane; }
};

// 64 rows of a [row][D] matrix into LDS, rows that are not there and columns from d on zero; flip: the last row first.  In whole pieces the loads
// go through a buffer that ends with the last row, straight into LDS; a thread's pieces lie a multiple of 16 rows apart, with which the swizzle
// repeats, so that one offset serves them all.
template <typename T, int D, bool VEC> struct LaStage {
  typedef LaTile<T, D> Tile;
  static constexpr int NT = LaWave<D>::NT, BYTES = LA_T * Tile::ROW, PIECES = BYTES / 16, N = PIECES / NT, EPP = 16 / (int)sizeof(T), RPN = NT / Tile::PPR;
  static_assert(PIECES % NT == 0 && RPN % 16 == 0, "whole pieces for every thread, the same swizzle for all of a thread's");
  uint32_t at;                     // of the piece with the lowest offset
  __device__ __forceinline__ void init(int64_t ld, int d, bool flip) {
    const int row = threadIdx.x / Tile::PPR, byte = ((threadIdx.x % Tile::PPR) ^ Tile::key(row)) * 16, from = flip ? RPN - 1 - row : row;
    at = byte < d * (int)sizeof(T) ? (uint32_t)(from * (int)ld) * (uint32_t)sizeof(T) + (uint32_t)byte : PK_OUT;
  }
  // src: the tile's first row in memory, rows: how many there are
  __device__ __forceinline__ void fetch(la_lds tile, const T* src, int64_t ld, int rows, int d, bool flip) const {
    rows = min(rows, LA_T);
    if constexpr (VEC) {
      const uint32_t bytes = (uint32_t)((rows - 1) * (int)ld + d) * (uint32_t)sizeof(T);
      const dma_i32x4 rs = dma_rsrc(src, bytes);
      const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)tile), step = (uint32_t)(RPN * (int)ld) * (uint32_t)sizeof(T);
      const uint32_t to = lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024u;
#pragma unroll
      for (int n = 0; n < N; ++n)                                // (PK_OUT and a few steps lie behind every such buffer too)
        dma_load(to + (uint32_t)n * NT * 16u, at + (uint32_t)(flip ? N - 1 - n : n) * step, rs);
    } else {
      union { piece_u4 u; T e[EPP]; } v;
#pragma unroll 1
      for (int n = 0; n < N; ++n) {
        const int q = n * NT + (int)threadIdx.x, row = q / Tile::PPR, byte = ((q % Tile::PPR) ^ Tile::key(row)) * 16, from = flip ? LA_T - 1 - row : row;
        const int c = byte / (int)sizeof(T);
        const T* p = src + (int64_t)from * ld + c;
        v.u = piece_u4{0, 0, 0, 0};
        if (from < rows) {
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
// zeros in the first n rows of two tiles that lie behind each other; barriers around it are the caller's
template <typename T, int D> __device__ __forceinline__ void la_clear(la_lds tile, int n) {
  typedef __attribute__((address_space(3))) pk_i4* la_i4;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    for (int i = (int)threadIdx.x * 16; i < n * LaTile<T, D>::ROW; i += LaWave<D>::NT * 16)
      *(la_i4)(tile + k * LA_T * LaTile<T, D>::ROW + i) = pk_i4{0, 0, 0, 0};
}
// until the loads into LDS have landed, for all wavefronts
template <bool VEC> __device__ __forceinline__ void la_land() {
  if constexpr (VEC) pk_landed();
  __syncthreads();
}

// Where a row's sequence begins, counted in the tile's rows in the order of the walk: -1 before the tile; this: in no sequence
constexpr int LA_NONE = LA_T;

// The sequences of a tile's rows from a lookup of LA_SPAN rows: a lane's row r of the tile (in memory) lies in [start, end).  Every
// word of the lookup is in a lane, the last one that begins before the tile and the first one behind it come out of two ballots.
struct LaSpan {
  uint32_t word;
  uint64_t some;                   // words that are not empty
  int t0, lo, hi, first, last;
  template <typename P> __device__ __forceinline__ void take(const P& pr, int t0_, int lane) {
    word = lane < LA_SPAN / 32 ? pr.mark[lane] : 0u;
    some = __ballot(word != 0);
    t0 = t0_;
    lo = __builtin_amdgcn_readfirstlane(pr.lo);
    hi = __builtin_amdgcn_readfirstlane(pr.hi);
    first = __builtin_amdgcn_readfirstlane(pr.first);
    last = __builtin_amdgcn_readfirstlane(pr.last);
  }
  // m0: the tile's first row, i: a row of it
  __device__ __forceinline__ bool range(int m0, int i, int& start, int& end) const {
    const int w = (m0 - t0) >> 5;
    const uint64_t marks = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)word, w + 1) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)word, w);
    const uint64_t before = some & ((1ull << w) - 1), behind = some >> (w + 2);
    int from = lo, to = hi;
    if (before) {
      const int k = 63 - __builtin_clzll(before);
      from = t0 + 32 * k + 31 - __builtin_clz((uint32_t)__builtin_amdgcn_readlane((int)word, k));
    }
    if (behind) {
      const int k = w + 2 + __builtin_ctzll(behind);
      to = t0 + 32 * k + __builtin_ctz((uint32_t)__builtin_amdgcn_readlane((int)word, k));
    }
    const uint64_t up = 2ull * ((1ull << i) - 1) + 1, at = marks & up, past = marks & ~up;       // bits 0 .. i, and the others
    start = at ? m0 + 63 - __builtin_clzll(at) : from;
    end = past ? m0 + __builtin_ctzll(past) : to;
    return m0 + i >= first && m0 + i < last;
  }
};

// bf16 pairs with infinities and NaNs have bit 15 of a half set in the result
__device__ __forceinline__ uint32_t la_odd(uint32_t u) { return (u & 0x7f807f80u) + 0x00800080u; }

typedef __attribute__((address_space(3))) pk_s4* la_lds4;
union LaFrag { uint32_t u[4]; pk_s4 h[2]; pk_bf8 v; bf16_raw e[8]; };

// Sixteen columns of a staged bf16 tile over 32 rows as a matrix operand: a lane's slots are rows row0 + 4 g + 0..3 and 16 + 4 g + 0..3; it holds
// column col0 + l.  `at`: la_cols_at(), row0: a multiple of 32, col0: of 16
template <int D> __device__ __forceinline__ uint32_t la_cols_at(int lane) {
  const int r = lane & 15;
  uint32_t a = (uint32_t)LaTile<bf16_raw, D>::at(4 * (lane >> 4) + (r >> 2), 4 * (r & 3) * 2);
  asm volatile("" : "+v"(a));                                    // (formed where it is needed)
  return a;
}
template <int D> __device__ __forceinline__ void la_cols(LaFrag& f, la_lds tile, uint32_t at, int row0, int col0) {
#pragma unroll
  for (int h = 0; h < 2; ++h)                                    // (sixteen rows on the swizzle repeats)
    f.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((la_lds4)(tile + (at ^ (uint32_t)(col0 << 1)) + (row0 + 16 * h) * LaTile<bf16_raw, D>::ROW));
}

// A state in the accumulators of the wavefronts: s[kt][i], column 16 cs + l of c, and of b
__device__ __forceinline__ int la_row(int kt, int i, int g) { return 16 * kt + 4 * g + i; }
// its place in a block's sums
template <int D> __device__ __forceinline__ la_f4* la_sum(float* sums, int cs, int kt, int lane) {
  return reinterpret_cast<la_f4*>(sums) + (cs * (D / 16) + kt) * 64 + lane;
}

// a pair of values as two bf16 words, value and rest; x becomes what is left of it
__device__ __forceinline__ uint32_t la_word(float& x0, float& x1) {
  const uint32_t u = pack_bf16x2(x0, x1);
  x0 -= __uint_as_float(u << 16);
  x1 -= __uint_as_float(u & 0xffff0000u);
  return u;
}

// s = a block's sum, or its transpose
template <typename T, int D> __device__ __forceinline__ void la_load_sum(la_f4 (&s)[D / 16], float* sum, bool turned, const LaWave<D>& wv) {
  if (!turned) {
#pragma unroll
    for (int kt = 0; kt < D / 16; ++kt) s[kt] = *la_sum<D>(sum, wv.cs, kt, wv.lane);
  } else {                                                       // entry (row, column) is (column, row) of what lies there
    const int c = 16 * wv.cs + wv.l;                             // the row there, and where it lies
    const float* p = sum + ((c >> 4) * 64 + 16 * (c >> 2 & 3)) * 4 + (c & 3);
#pragma unroll
    for (int kt = 0; kt < D / 16; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = la_row(kt, i, wv.g);
        s[kt][i] = p[((r >> 4) * (D / 16) * 64 + (r & 15)) * 4];
      }
  }
}

// which of rows r and r + 1 lie in [c0, c1), as a mask of two halves
__device__ __forceinline__ uint32_t la_rows(int r, int c0, int c1) {
  return (r >= c0 && r < c1 ? 0xffffu : 0u) | (r + 1 >= c0 && r + 1 < c1 ? 0xffff0000u : 0u);
}

// s += sum over tile rows of w[row] b[row]^T c[row], w: LDS.  PART: rows outside of [c0, c1), whose weights are zero, may hold anything.
// THREE: c w as three words
template <typename T, int D, bool PART, bool THREE>
__device__ __forceinline__ void la_update(la_f4 (&s)[D / 16], la_lds tb, la_lds tc, const float* w, int c0, int c1, const LaWave<D>& wv) {
  const int lane = wv.lane, g = wv.g;
  int g4 = 4 * g;
  if constexpr (PART) asm volatile("" : "+v"(c0), "+v"(c1), "+v"(g4));      // (masks are formed where they are needed)
  if constexpr (sizeof(T) == 2) {
    const uint32_t at = la_cols_at<D>(lane);
#pragma unroll
    for (int ks = 0; ks < LA_T / 32; ++ks) {
      const int row0 = 32 * ks;
      LaFrag c, hi, lo, ll;
      la_cols<D>(c, tc, at, row0, 16 * wv.cs);
      const float4 w0 = *reinterpret_cast<const float4*>(w + row0 + 4 * g), w1 = *reinterpret_cast<const float4*>(w + row0 + 16 + 4 * g);
      const float wt[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
      if constexpr (PART) {                                      // zeros in the rows that do not take part
#pragma unroll
        for (int p = 0; p < 4; ++p) c.u[p] &= la_rows(row0 + g4 + 2 * (p & 1) + 16 * (p >> 1), c0, c1);
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float x0 = __uint_as_float(c.u[p] << 16) * wt[2 * p], x1 = __uint_as_float(c.u[p] & 0xffff0000u) * wt[2 * p + 1];
        hi.u[p] = la_word(x0, x1);
        lo.u[p] = la_word(x0, x1);
        if constexpr (THREE) ll.u[p] = la_word(x0, x1);
      }
#pragma unroll
      for (int k0 = 0; k0 < D / 16; k0 += 2) {                   // (four of b's columns' reads at once would take the registers of the state)
        LaFrag b[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          la_cols<D>(b[k], tb, at, row0, 16 * (k0 + k));
          if constexpr (PART) {
#pragma unroll
            for (int p = 0; p < 4; ++p) b[k].u[p] &= la_rows(row0 + g4 + 2 * (p & 1) + 16 * (p >> 1), c0, c1);
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) s[k0 + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[k].v, hi.v, s[k0 + k], 0, 0, 0);
#pragma unroll
        for (int k = 0; k < 2; ++k) s[k0 + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[k].v, lo.v, s[k0 + k], 0, 0, 0);
        if constexpr (THREE) {
#pragma unroll
          for (int k = 0; k < 2; ++k) s[k0 + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[k].v, ll.v, s[k0 + k], 0, 0, 0);
        }
        if (k0 % 4 == 2) __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    typedef LaTile<T, D> Tile;
    uint32_t at = (uint32_t)Tile::at(4 * g, wv.l * 4);           // row 16 ks + 4 g + i: other bits of the key
    asm volatile("" : "+v"(at));
#pragma unroll 1
    for (int ks = 0; ks < LA_T / 16; ++ks) {
      const float4 w4 = *reinterpret_cast<const float4*>(w + 16 * ks + 4 * g);
      const float wt[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 16 * ks + 4 * g + i;
        const uint32_t to = (uint32_t)(16 * ks + i) * Tile::ROW, key = (uint32_t)Tile::key(i) << 4;
        const bool out = PART && (row < c0 || row >= c1);
        float c = *(__attribute__((address_space(3))) const float*)(tc + (at ^ (key ^ (uint32_t)(wv.cs << 6))) + to) * wt[i];
        if (out) c = 0.f;
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) {
          float b = *(__attribute__((address_space(3))) const float*)(tb + (at ^ (key ^ (uint32_t)(kt << 6))) + to);
          if (out) b = 0.f;
          s[kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(b, c, s[kt], 0, 0, 0);
        }
      }
    }
  }
}

// a sequence's state from and to memory
template <typename T, int D> __device__ __forceinline__ int64_t la_state_at(const LaArgs& a, int b, int seq, int hk) {
  return (((int64_t)b * a.nseq + seq) * a.Hkv + hk) * a.d * a.d;
}
template <typename T, int D>
__device__ __forceinline__ void la_load_state(la_f4 (&s)[D / 16], const LaJob& J, const LaArgs& a, int b, int seq, int hk, const LaWave<D>& wv) {
  const float* p = J.S0 + la_state_at<T, D>(a, b, seq, hk);
  int col = 16 * wv.cs + wv.l;
  asm volatile("" : "+v"(col));
  const int rs = J.flip ? 1 : a.d, cs = J.flip ? a.d : 1;
  const float f = 1.f / J.fi;
  const float* pc = p + min(col, a.d - 1) * cs;                  // (loads that are all made: a branch around each would wait for each)
#pragma unroll
  for (int kt = 0; kt < D / 16; ++kt)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[kt][i] = pc[min(la_row(kt, i, wv.g), a.d - 1) * rs];
#pragma unroll
  for (int kt = 0; kt < D / 16; ++kt)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[kt][i] = la_row(kt, i, wv.g) < a.d && col < a.d ? f * s[kt][i] : 0.f;
}
template <typename T, int D> __device__ __forceinline__ void la_store_state(const la_f4 (&s)[D / 16], float* p, int d, float f, const LaWave<D>& wv) {
  int col = 16 * wv.cs + wv.l;
  asm volatile("" : "+v"(col));
#pragma unroll
  for (int kt = 0; kt < D / 16; ++kt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = la_row(kt, i, wv.g);
      if (row < d && col < d) p[row * d + col] = f * s[kt][i];
    }
}
// which sequence a row belongs to: the last one that begins at or before it, sixty-four places a step (every lane the same row)
__device__ __forceinline__ int la_sequence(const int32_t* off, int nseq, int r) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  for (int n = nseq; n > 1;) {
    const int step = (n + 63) >> 6;
    const int le = __popcll(__ballot(lane * step < n && off[min(lo + lane * step, nseq - 1)] <= r));
    const int skip = max(le - 1, 0) * step;
    lo += skip;
    n = min(step, n - skip);
  }
  return lo;
}

// s times what `f` (la_faded) stands for, the same in all lanes
template <int N> __device__ __forceinline__ void la_fade(la_f4 (&s)[N], float f) {
  f = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(f)));
  if (f > 0.f) {
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] *= f;
  }
  asm volatile("" : "+s"(f));                                    // (two branches: as one, its ends would take registers of their own)
  if (!(f > 0.f)) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] = fmaf(s[n][i], f, s[n][i]);
  }
}

// every line of a launch's arguments at once: what is looked up in them by the job would wait for each of them in turn
__device__ __forceinline__ void la_touch(const LaArgs& a) {
  const uint32_t* p = reinterpret_cast<const uint32_t*>(&a);
  static_assert(sizeof(LaArgs) > 640 && sizeof(LaArgs) <= 704, "eleven lines");
  asm volatile("" ::"s"(p[0]), "s"(p[16]), "s"(p[32]), "s"(p[48]), "s"(p[64]), "s"(p[80]), "s"(p[96]), "s"(p[112]), "s"(p[128]), "s"(p[144]), "s"(p[160]));
}

// Workgroup -> (job, model, head of the job, block).  Jobs with as many heads as each other take turns, eight workgroups each, so that a head's and
// block's jobs, which read the same tiles, follow each other on the same XCD.
struct LaPlace {
  int job, b, h, blk;
  bool none;                       // past the last place
  __device__ __forceinline__ LaPlace(const LaArgs& a, bool key_heads) {
    uint32_t x = blockIdx.x;
    job = 0;
    PkDiv by = key_heads ? a.by_key_heads : a.by_heads;          // (B times heads, heads)
    PkDiv of = key_heads ? a.by_hkv : a.by_hq;
    uint32_t n = (uint32_t)a.blocks * by.d;
    if (key_heads) {
      while (x >= n && job < a.nsums - 1) { x -= n; ++job; }
    } else {
      const int turns = a.jobs == 1 ? 1 : a.by_hq.d == a.by_hkv.d ? 3 : 2;       // jobs that take turns: all, or the last two
      if (a.jobs == 3 && turns == 2) {
        if (x < n) {
          turns_of(x, 1);
        } else {
          x -= n;
          by = a.by_key_heads;
          of = a.by_hkv;
          n = (uint32_t)a.blocks * by.d;
          turns_of(x, 2);
          ++job;
        }
      } else {
        turns_of(x, turns);
      }
    }
    none = x >= n;
    const uint32_t k = by(x), bh = x - k * by.d;
    blk = (int)k;
    b = (int)of(bh);
    h = (int)(bh - (uint32_t)b * of.d);
  }
  __device__ __forceinline__ void turns_of(uint32_t& x, int turns) {
    if (turns == 1) return;
    const uint32_t eight = x >> 3, q = turns == 2 ? eight >> 1 : eight / 3u;
    job = (int)(eight - q * (uint32_t)turns);
    x = q << 3 | (x & 7);
  }
  // workgroups in all
  static int64_t count(const LaArgs& a, bool key_heads) {
    const int64_t k = (int64_t)a.blocks * a.by_key_heads.d, q = (int64_t)a.blocks * a.by_heads.d, k8 = (k + 7) / 8 * 8, q8 = (q + 7) / 8 * 8;
    return key_heads ? k * a.nsums : a.jobs == 1 ? q : a.by_hq.d == a.by_hkv.d ? 3 * q8 : q + 2 * k8;
  }
};

}  // namespace hfta
