// Attention over packed sequences of different lengths with grouped heads, forward and backward (fusion rules table row
// "MultiheadAttention": the projections are fused Linears, this is what stands between them).
//
//   x_ij = scale q_i . k_j for j in i's sequence (causal: j <= i),  lse_i = log sum_j exp x_ij,  p_ij = exp(x_ij - lse_i)
//   ctx_i = sum_j p_ij v_j
//   D_i = dctx_i . ctx_i,  ds_ij = p_ij (dctx_i . v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij dctx_i   (i: all heads of the group)
//
// Nothing of the size of the scores is stored.  Forward: one pass over the keys with the running maximum and sum of the
// softmax; lse is all that the backward needs to form p again.  Backward: two kernels, one per side that owns its sums
// (a query tile its dq, a key tile its dk and dv over all heads of the group), so that there are no atomics and results
// are the same bit for bit on every run; scores are formed twice for that (14 instead of 10 products of d per pair).
//
// A tile is a stretch of the packed rows, whatever sequences it holds: the keys that its rows see are one stretch again,
// because sequences are contiguous.  Many short sequences share a tile, and nothing is planned on the host.
//
// Matrix instruction 32 x 32: with the keys as its first operand a lane holds one query (l%32) and sixteen keys
// 8(i/4) + 4(l/32) + i%4, so a row's softmax needs one exchange between two lanes, and the result is the second operand
// of the product over keys if the other side orders its keys the same way (slots 0..3 of a lane half: keys 4g + 0..3,
// slots 4..7: 8 + 4g + 0..3).  For bf16 that order is what two LDS transpose reads deliver.  fp32 takes the fp32
// instruction, whose operands are single values per lane.
//
// Entries outside a row's sequence are taken out of the scores by a select, so what stands there does not matter, but
// in the product over keys a zero probability times a NaN or an infinity would be a NaN.  Products are therefore made
// as if all values were finite; if a result is not, the workgroup does its rows again, with those values zero in the
// product over keys and NaN put into what they belong to in the rows that do see them.
//
// A workgroup is four wavefronts.  With many rows each takes 32 rows of its own and all keys, which the workgroup stages 64
// at a time, twice buffered with one barrier per tile.  Where that leaves compute units without work (SPLIT), all four take the
// same 32 rows and a quarter of the key blocks each, from LDS of their own without barriers, and join at the end.
//
// Measured, bf16: forward of 16384 rows in two sequences, 8 heads of 128 over 2, 313 us (943 TFLOP/s; a library product of 8192^3 reaches
// 1198): bound by the vector work of the softmax beside the matrix instructions.  2 x 8192 rows in three, the same heads: forward 153,
// queries' backward 205, keys' 358 and 28 for its parts, the last bound by registers.  8 x 2048 rows in twelve, 4 heads of 64: 17, 21 and 26 us,
// chains of a few tiles at 1.6 to 2 us each; bytes alone would be 14.
#pragma once
#include "gemm_dma.h"
#include "packed_rows.h"

#include <math.h>
#include <type_traits>

namespace hfta {

typedef __bf16 pk_bf8 __attribute__((ext_vector_type(8)));
typedef float pk_f16 __attribute__((ext_vector_type(16)));
typedef short pk_s4 __attribute__((ext_vector_type(4)));

constexpr int PK_WT = 32;                                        // rows of a wavefront
constexpr float PK_LOG2E = 1.4426950408889634f, PK_LN2 = 0.6931471805599453f;

struct PkStr { int64_t b, r, h; };
// x / d for x < 2^31 by a product (d >= 1): m = floor(2^(31 + l) / d) + 1 with l = ceil(log2 d) is off by at most 1 / 2^(31 + l) d per unit of x
struct PkDiv {
  uint32_t d, m, s;
  PkDiv() = default;
  explicit PkDiv(uint32_t x) : d(x), m(0), s(0) {
    while ((1ull << s) < x) ++s;
    m = (uint32_t)((1ull << (31 + s)) / x + 1);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)(((uint64_t)x * m) >> 31 >> s); }
};
struct PkArgs {
  const void *Q, *K, *V, *dCTX;
  const int32_t* off;
  void *CTX, *dQ, *dK, *dV;
  float *LSE, *Dsum, *part;        // Dsum, part: the backward's workspace
  PkStr qs, ks, cs, dqs, dks;
  int B, R, nseq, Hq, Hkv, d, causal, parts;       // parts: workgroups that share the sums of a tile of keys
  int twice;                       // sequences are short: the queries' backward sums D's rest first
  PkDiv by_heads, by_hkv, by_group, by_parts;      // B Hkv, Hkv, Hq / Hkv, parts
  float scale;
};
constexpr int PK_PARTS_MAX = 8;
struct PkForm { bool bf16, vec, split; };                        // storage, rows in 16-byte pieces, keys split over wavefronts
int pk_fwd(const PkArgs& a, const PkForm& f, hipStream_t st);    // attention_packed_fwd.hip
int pk_dq(const PkArgs& a, const PkForm& f, hipStream_t st);     // attention_packed_dq.hip
int pk_dkv(const PkArgs& a, const PkForm& f, hipStream_t st);    // attention_packed_dkv.hip

constexpr float PK_SLACK = 8.f;
// of a lane and the one 32 on
__device__ __forceinline__ float pk_both_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pk_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// A staged tile: rows of D columns without padding, as the loads into LDS leave them; piece p (16 bytes) of row r lies at place p ^ key(r).
// Sixteen rows' reads of one piece then cover all 64 banks once, and so do a transpose read's four rows of four pieces.
template <typename T, int D> struct PkTile {
  static constexpr int ROW = D * (int)sizeof(T), PPR = ROW / 16;
  static __device__ __forceinline__ constexpr int key(int r) {
    return PPR >= 16 ? (r & 3) << 2 | (r >> 2 & 3) : PPR == 8 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : r >> 2 & 3;
  }
  static __device__ __forceinline__ int at(int r, int byte) { return r * ROW + (((byte >> 4) ^ key(r)) << 4) + (byte & 15); }
};

// ------------------------------------------------------------------ operands
// A lane's row (l%32) of a 32 x D matrix as the second operand of a product over columns.
template <typename T, int D> struct PkRow;
template <int D> struct PkRow<bf16_raw, D> {
  static constexpr int N = D / 16, STEP = 16, EPP = 8;
  union Piece { uint4 u; pk_bf8 v; bf16_raw e[8]; };
  Piece p[N];                                                    // columns 16 s + 8 (l/32) + 0..7
};
template <int D> struct PkRow<float, D> {
  static constexpr int N = D / 8, STEP = 8, EPP = 4;
  union Piece { uint4 u; float e[4]; };
  Piece p[N];                                                    // columns 8 s + 4 (l/32) + 0..3
};

template <typename T, int D, bool VEC>
__device__ __forceinline__ void pk_load_row(PkRow<T, D>& x, const T* row, bool ok, int d, int g) {
#pragma unroll
  for (int s = 0; s < PkRow<T, D>::N; ++s) {
    const int c = s * PkRow<T, D>::STEP + g * PkRow<T, D>::EPP;
    x.p[s].u = make_uint4(0, 0, 0, 0);
    if constexpr (VEC) {
      if (ok && c < d) x.p[s].u = *reinterpret_cast<const uint4*>(row + c);
    } else {
#pragma unroll
      for (int e = 0; e < PkRow<T, D>::EPP; ++e)
        if (ok && c + e < d) x.p[s].e[e] = row[c + e];
    }
  }
}

// What follows in the code up to the next branch: AHEAD reads of LDS first, then MFMAS times one matrix instruction and PER reads.  Left to
// itself the compiler keeps two reads in flight, and each pair's latency shows.
template <int AHEAD, int MFMAS, int PER> __device__ __forceinline__ void pk_order() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < MFMAS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
  }
}

// acc[n][tile row][lane row] = sum over columns of tile row row0 + 32 n + .. (row0: a multiple of 32) and the lane's row x
template <typename T, int D, int NB>
__device__ __forceinline__ void pk_rows(pk_f16 (&acc)[NB], const unsigned char* tile, int row0, const PkRow<T, D>& x, int lane) {
  typedef PkTile<T, D> Tile;
  const uint32_t a = (uint32_t)((lane & 31) * Tile::ROW + (((lane >> 5) ^ Tile::key(lane & 31)) << 4));
  const unsigned char* t = tile + row0 * Tile::ROW;
#pragma unroll
  for (int s = 0; s < PkRow<T, D>::N; ++s)                       // two pieces of the tile's row, one for each half of the lanes
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const unsigned char* p = t + (a ^ (uint32_t)(s << 5)) + n * 32 * Tile::ROW;
      if constexpr (sizeof(T) == 2) {
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const pk_bf8*>(p), x.p[s].v, acc[n], 0, 0, 0);
      } else {
        const float4 v = *reinterpret_cast<const float4*>(p);
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.x, x.p[s].e[0], acc[n], 0, 0, 0);
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.y, x.p[s].e[1], acc[n], 0, 0, 0);
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.z, x.p[s].e[2], acc[n], 0, 0, 0);
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.w, x.p[s].e[3], acc[n], 0, 0, 0);
      }
    }
}

// A product over 32 tile rows: acc[c/32][column c of the tile][lane row] += sum of tile[row0 + i][c] w[i], where w holds
// the weights as a product's result does.
template <typename T, int D>
__device__ __forceinline__ void pk_cols(pk_f16 (&acc)[D / 32], const unsigned char* tile, int row0, const pk_f16& w, int lane) {
  typedef PkTile<T, D> Tile;
  const int g = lane >> 5;
  const unsigned char* t0 = tile + row0 * Tile::ROW;
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) pk_s4* lds_s4;
    union Frag { uint32_t u[4]; pk_s4 h[2]; pk_bf8 v; } f, x;
    const int r = lane & 15, row = 4 * g + (r >> 2);
    const uint32_t a = (uint32_t)Tile::at(row, (16 * ((lane >> 4) & 1) + 4 * (r & 3)) * 2);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f.u[e] = pack_bf16x2(w[8 * t + 2 * e], w[8 * t + 2 * e + 1]);
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) {
#pragma unroll
        for (int h = 0; h < 2; ++h)                              // eight rows on: another bit of the key
          x.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(t0 + (a ^ (uint32_t)(cb << 6 | h << 5)) + (16 * t + 8 * h) * Tile::ROW));
        acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v, f.v, acc[cb], 0, 0, 0);
      }
    }
  } else {
    const uint32_t a = (uint32_t)Tile::at(4 * g, (lane & 31) * 4);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      constexpr int ROW = Tile::ROW;
      const int row = 8 * (i >> 2) + (i & 3);                    // (past 4 g: the other bits of the key)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
        acc[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(t0 + (a ^ (uint32_t)(Tile::key(row) << 4 ^ cb << 7)) + row * ROW),
                                                       w[i], acc[cb], 0, 0, 0);
    }
  }
}

// Tile rows j0 + .. (of the tensor) at row0 of the tile: NaN for the entries that a value which is not finite takes part in,
// in lane rows that see its row, [lo, hi).
template <typename T, int D>
__device__ __forceinline__ void pk_mark(pk_f16 (&acc)[D / 32], const unsigned char* tile, int row0, int j0, int lo, int hi, int lane) {
  typedef PkTile<T, D> Tile;
#pragma unroll 1
  for (int r = 0; r < 32; ++r) {
    const bool sees = j0 + r >= lo && j0 + r < hi;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = cb * 32 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
        const float x = Elem<T>::load(reinterpret_cast<const T*>(tile + Tile::at(row0 + r, c * (int)sizeof(T)))), y = sees ? x : 0.f;
        acc[cb][i] += y - y;                                     // NaN, or nothing
      }
  }
}

// ------------------------------------------------------------------ tiles
// until none of this wavefront's loads is in flight
__device__ __forceinline__ void pk_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Rows of a [row][D] matrix into LDS, a workgroup's 64 or 32 or (SPLIT) a wavefront's 32; rows that are not there and columns
// from d on: zeros.  fetch() starts the loads of a tile and land() ends them; the tile's place must not be read in between.
// In whole pieces the loads go through a buffer that ends with the last row, which gives the zeros; it is placed anew for
// every tile, so that offsets stay small however far the rows lie.  A workgroup's tile is loaded into LDS itself, without
// registers (32 of 256 at d = 128); the others pass through them.
typedef int pk_i4 __attribute__((ext_vector_type(4)));
constexpr int64_t PK_LD_MAX = 1 << 22;                           // elements between rows that such a buffer's offsets take
constexpr uint32_t PK_OUT = 0x80000000u;                         // an offset past every such buffer
template <typename T, int D, bool VEC, bool SPLIT, int TILE = 64> struct PkStage {
  static constexpr int ROWS = SPLIT ? 32 : TILE, NT = SPLIT ? 64 : 256, BYTES = ROWS * PkTile<T, D>::ROW, PIECES = BYTES / 16;
  static constexpr int PPR = PkTile<T, D>::PPR, N = (PIECES + NT - 1) / NT, EPP = 16 / (int)sizeof(T);
  static constexpr bool DIRECT = VEC && !SPLIT;
  union Piece { pk_i4 i; uint4 u; T e[EPP]; uint32_t w[4]; };
  typename std::conditional<DIRECT, uint32_t, Piece>::type v[N]; // offsets of a lane's pieces, or the pieces
  static __device__ __forceinline__ int tid() { return SPLIT ? threadIdx.x & 63 : threadIdx.x; }
  // row and source byte of a thread's n-th place
  static __device__ __forceinline__ void place(int n, int& row, int& byte) {
    const int q = n * NT + tid();
    row = q / PPR;
    byte = ((q % PPR) ^ PkTile<T, D>::key(row)) * 16;
  }
  static __device__ __forceinline__ uint32_t offset(int n, int64_t ld, int d) {
    int row, byte;
    place(n, row, byte);
    return row < ROWS && byte < d * (int)sizeof(T) ? (uint32_t)(row * (int)ld) * (uint32_t)sizeof(T) + (uint32_t)byte : PK_OUT;
  }
  __device__ __forceinline__ void init(int64_t ld, int d) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = offset(n, ld, d);
    }
  }
  // src: the tile's first row, rows: how many there are; the same for all threads that share the tile
  __device__ __forceinline__ void fetch(unsigned char* tile, const T* src, int64_t ld, int rows, int d) {
    const uint32_t bytes = rows > 0 ? (uint32_t)((min(rows, ROWS) - 1) * (int)ld + d) * (uint32_t)sizeof(T) : 0u;
    if constexpr (DIRECT) {
      const dma_i32x4 rs = dma_rsrc(src, bytes);
      const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)tile);
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int n = 0; n < N; ++n)
        if ((n * NT + wave * 64) < PIECES) dma_load(lds + (uint32_t)(n * NT + wave * 64) * 16u, v[n], rs);
    } else if constexpr (VEC) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(src), 0, (int)bytes, 0x00020000);
#pragma unroll
      for (int n = 0; n < N; ++n) v[n].i = __builtin_amdgcn_raw_buffer_load_b128(rs, offset(n, ld, d), 0, 0);
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        int row, byte;
        place(n, row, byte);
        const int c = byte / (int)sizeof(T);
        const T* p = src + (int64_t)row * ld + c;
        v[n].u = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < EPP; ++e)
          if (row < min(rows, ROWS) && c + e < d) v[n].e[e] = p[e];
      }
    }
  }
  __device__ __forceinline__ void land(unsigned char* tile) const {
    if constexpr (DIRECT) {
      pk_landed();
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (n * NT + tid() < PIECES) *reinterpret_cast<uint4*>(tile + (n * NT + tid()) * 16) = v[n].u;
    }
  }
  static __device__ __forceinline__ void clean(unsigned char* tile, int rows) {      // zeros in place of values that are not finite
    for (int q = tid(); q < rows * PPR; q += NT) {
      Piece x;
      x.u = *reinterpret_cast<const uint4*>(tile + q * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
          if ((x.w[e] & 0x7f80u) == 0x7f80u) x.w[e] &= 0xffff0000u;
          if ((x.w[e] & 0x7f800000u) == 0x7f800000u) x.w[e] &= 0xffffu;
        } else {
          if ((x.w[e] & 0x7f800000u) == 0x7f800000u) x.w[e] = 0;
        }
      }
      *reinterpret_cast<uint4*>(tile + q * 16) = x.u;
    }
  }
};
// 32 values from src, of which `rows` are there, to LDS, by lanes 0..31
__device__ __forceinline__ void pk_fetch32(float* lds, const float* src, int rows, int lane) {
  const dma_i32x4 rs = dma_rsrc(src, rows > 0 ? (uint32_t)min(rows, 32) * 4u : 0u);
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) float*)lds);
  if (lane < 32)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(at), "v"((uint32_t)lane * 4u), "s"(rs) : "memory", "m0");
}
// between writing a tile and reading it: all wavefronts, or the lanes of one
template <bool SPLIT> __device__ __forceinline__ void pk_sync() {
  if constexpr (SPLIT) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  else __syncthreads();
}

// a lane's row of a result: columns 32 cb + 8 (i/4) + 4 (l/32) + i%4, column blocks from cb0 on
template <typename T, int NCB, bool VEC>
__device__ __forceinline__ void pk_store_row(T* row, const pk_f16 (&acc)[NCB], float f, int cb0, int d, int g) {
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = (cb0 + cb) * 32 + q * 8 + 4 * g;
      const float x[4] = {f * acc[cb][4 * q], f * acc[cb][4 * q + 1], f * acc[cb][4 * q + 2], f * acc[cb][4 * q + 3]};
      if constexpr (VEC) {
        if (c >= d) continue;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(row + c) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        else *reinterpret_cast<float4*>(row + c) = make_float4(x[0], x[1], x[2], x[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < d) Elem<T>::store(row + c + e, x[e]);
      }
    }
}

template <int N> __device__ __forceinline__ bool pk_not_finite(const pk_f16 (&acc)[N]) {
  float z = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = fmaf(0.f, acc[n][i], z);
  return z != z;
}

// The four wavefronts' sums of the same rows, added in order: wavefront w gets column block w (w < D / 32) in acc[0].  lds: 512 D bytes.
template <int D> __device__ __forceinline__ void pk_join(pk_f16 (&acc)[D / 32], float* lds, int wave, int lane) {
  __syncthreads();                                               // the tiles that lay there have been read
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) lds[((wave * (D / 32) + cb) * 16 + i) * 64 + lane] = acc[cb][i];
  __syncthreads();
  if (wave < D / 32) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float* x = lds + (wave * 16 + i) * 64 + lane;
      constexpr int W = D / 32 * 1024;
      acc[0][i] = (x[0] + x[W]) + (x[2 * W] + x[3 * W]);
    }
  }
}

template <typename T> __device__ __forceinline__ const T* pk_at(const void* p, const PkStr& s, int b, int h) {
  return reinterpret_cast<const T*>(p) + b * s.b + h * s.h;
}
template <typename T> __device__ __forceinline__ T* pk_at(void* p, const PkStr& s, int b, int h) {
  return reinterpret_cast<T*>(p) + b * s.b + h * s.h;
}

// Workgroup -> (tile, key head, head of its group).  Key heads run fastest, so that where their number is a multiple of
// eight all workgroups that read one head's keys share an XCD's L2.  The last tiles, of which rows see the most keys where
// attention is causal, come first; the first tiles do, of which keys are seen by the most rows (KEYS).
template <bool SPLIT> constexpr int pk_bm() { return SPLIT ? PK_WT : 4 * PK_WT; }
static inline int pk_tiles(int R, int bm) { return R / bm + (R % bm != 0); }
template <int BM, bool KEYS> struct PkPlace {
  int b, hk, hq, t0, part;         // KEYS: hq the group's first head
  __device__ __forceinline__ PkPlace(const PkArgs& a) {
    const uint32_t outer = a.by_heads(blockIdx.x), kh = blockIdx.x - outer * a.by_heads.d;       // of all key heads
    const PkDiv& by = KEYS ? a.by_parts : a.by_group;
    const uint32_t tile = by(outer), tiles = by(a.by_heads(gridDim.x));
    part = (int)(outer - tile * by.d);
    b = (int)a.by_hkv(kh);
    hk = (int)kh - b * a.Hkv;
    hq = hk * (int)a.by_group.d + (KEYS ? 0 : part);
    t0 = (int)(KEYS ? tile : tiles - 1 - tile) * BM;
  }
};

// The rows of a workgroup: what each sees of the other side ([lo, hi), empty outside the sequences), what the workgroup
// and the wavefront see together, and what all rows of the wavefront see.  Both ends grow with the row, so the first and the last
// row tell.
template <int BM> struct PkSpan {
  int row, lo, hi;
  bool in;
  int glo, ghi, wlo, whi, alo, ahi;
  // queries: keys from the sequence's start; keys: queries up to the sequence's end
  template <bool KEYS> static __device__ __forceinline__ bool ends(const PackedRows<BM>& pr, int causal, int t0, int i, int& lo, int& hi) {
    const bool in = pr.range(t0, i, lo, hi);
    if (causal && in) {
      if (KEYS) lo = t0 + i;
      else hi = t0 + i + 1;
    }
    return in;
  }
  // row0: the wavefront's first row in the tile
  template <bool KEYS> __device__ __forceinline__ void init(PackedRows<BM>& pr, const PkArgs& a, int b, int t0, int row0) {
    pr.template scan<256>(a.off + (int64_t)b * (a.nseq + 1), a.nseq, a.R, t0);
    const int i = row0 + (threadIdx.x & 31), f = max(pr.first - t0, 0), l = min(pr.last - t0, BM) - 1;
    row = t0 + i;
    in = ends<KEYS>(pr, a.causal, t0, i, lo, hi);
    glo = 0x7fffffff;
    ghi = 0;
    int x;
    if (f <= l) {
      ends<KEYS>(pr, a.causal, t0, f, glo, x);
      ends<KEYS>(pr, a.causal, t0, l, x, ghi);
    }
    glo = __builtin_amdgcn_readfirstlane(glo);
    ghi = __builtin_amdgcn_readfirstlane(ghi);
    const uint32_t m = (uint32_t)__ballot(in);
    wlo = 0x7fffffff;
    whi = alo = 0;
    ahi = 0x7fffffff;
    if (m) {
      const int fl = __builtin_ctz(m), ll = 31 - __builtin_clz(m);
      wlo = __builtin_amdgcn_readlane(lo, fl);
      ahi = __builtin_amdgcn_readlane(hi, fl);
      alo = __builtin_amdgcn_readlane(lo, ll);
      whi = __builtin_amdgcn_readlane(hi, ll);
    }
  }
  __device__ __forceinline__ bool none(int j0, int n) const { return j0 >= whi || j0 + n <= wlo; }      // of rows j0 .. j0 + n - 1
  // `none` in place of the entries i of s, tile rows j0 + 8(i/4) + 4g + i%4, that this lane's row does not see: a comparison with a
  // constant each, on the sides where a row of the wavefront has an end
  __device__ __forceinline__ void mask(pk_f16& s, int j0, int g, float none) const {
    if (j0 < alo) {
      const int x = lo - j0 - 4 * g;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) < x) s[i] = none;
    }
    if (j0 + 32 > ahi) {
      const int x = hi - j0 - 4 * g;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) >= x) s[i] = none;
    }
  }
};

// launch<T, D>(a, f, st) of the storage type and the tile's columns
#define PK_BY_SIZE(launch)                                                                                                            \
  (f.bf16 ? (a.d <= 32 ? launch<bf16_raw, 32>(a, f, st) : a.d <= 64 ? launch<bf16_raw, 64>(a, f, st) : launch<bf16_raw, 128>(a, f, st)) \
          : (a.d <= 32 ? launch<float, 32>(a, f, st) : a.d <= 64 ? launch<float, 64>(a, f, st) : launch<float, 128>(a, f, st)))

}  // namespace hfta
