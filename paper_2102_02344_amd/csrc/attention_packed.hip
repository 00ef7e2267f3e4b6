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
// as if all values were finite; if a result is not, the workgroup does its tile again with those values taken out of the
// product and added, as NaN, to the rows that do see them.
#include "packed_rows.h"

#include <math.h>

namespace hfta {
namespace {

typedef __bf16 pk_bf8 __attribute__((ext_vector_type(8)));
typedef float pk_f16 __attribute__((ext_vector_type(16)));
typedef short pk_s4 __attribute__((ext_vector_type(4)));

constexpr int PK_KT = 64;            // rows of a staged tile
constexpr int PK_WT = 32;            // rows of a wavefront
constexpr int PK_BM = 4 * PK_WT;     // rows of a workgroup
constexpr float PK_LOG2E = 1.4426950408889634f, PK_LN2 = 0.6931471805599453f;

template <typename T, int D> struct PkTile {
  static constexpr int PITCH = D * (int)sizeof(T) + 16;          // 16 rows' 16-byte reads cover all banks
  static constexpr int BYTES = PK_KT * PITCH;
};

__device__ __forceinline__ float pk_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// ------------------------------------------------------------------ operands
// A lane's row (l%32) of a 32 x D matrix as the second operand of a product over columns.
template <typename T, int D> struct PkRow;
template <int D> struct PkRow<bf16_raw, D> {
  static constexpr int N = D / 16;
  union Piece { uint4 u; pk_bf8 v; bf16_raw e[8]; };
  Piece p[N];                                                    // columns 16 s + 8 (l/32) + 0..7
  static constexpr int STEP = 16, EPP = 8;
};
template <int D> struct PkRow<float, D> {
  static constexpr int N = D / 8;
  union Piece { uint4 u; float e[4]; };
  Piece p[N];                                                    // columns 8 s + 4 (l/32) + 0..3
  static constexpr int STEP = 8, EPP = 4;
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

// acc[tile row][lane row] = sum over columns of tile row row0 + .. and the lane's row x
template <int D>
__device__ __forceinline__ void pk_rows(pk_f16& acc, const unsigned char* tile, int row0, const PkRow<bf16_raw, D>& x, int lane) {
  const unsigned char* a = tile + (row0 + (lane & 31)) * PkTile<bf16_raw, D>::PITCH + (lane >> 5) * 16;
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const pk_bf8*>(a + s * 32), x.p[s].v, acc, 0, 0, 0);
}
template <int D>
__device__ __forceinline__ void pk_rows(pk_f16& acc, const unsigned char* tile, int row0, const PkRow<float, D>& x, int lane) {
  const unsigned char* a = tile + (row0 + (lane & 31)) * PkTile<float, D>::PITCH + (lane >> 5) * 16;
#pragma unroll
  for (int s = 0; s < D / 8; ++s) {
    const float4 v = *reinterpret_cast<const float4*>(a + s * 32);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.x, x.p[s].e[0], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.y, x.p[s].e[1], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.z, x.p[s].e[2], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v.w, x.p[s].e[3], acc, 0, 0, 0);
  }
}

// A product over 32 tile rows: acc[c/32][column c of the tile][lane row] += sum of tile[row0 + i][c] w[i], where w holds
// the weights as a product's result does.  `safe`: values that are not finite are left out, and make NaN of the entries
// for which `seen` (bit i: the lane's row sees row i of the tile) holds.
template <int D, bool SAFE>
__device__ __forceinline__ void pk_cols(pk_f16 (&acc)[D / 32], const unsigned char* tile, int row0, const pk_f16& w, uint32_t seen,
                                        int lane) {
  constexpr int PITCH = PkTile<bf16_raw, D>::PITCH;
  typedef __attribute__((address_space(3))) pk_s4* lds_s4;
  union Frag { uint32_t u[4]; pk_s4 h[2]; pk_bf8 v; } f, x;
  const int g = lane >> 5, r = lane & 15;
  const unsigned char* a = tile + (row0 + 4 * g + (r >> 2)) * PITCH + (16 * ((lane >> 4) & 1) + 4 * (r & 3)) * 2;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f.u[e] = pack_bf16x2(w[8 * t + 2 * e], w[8 * t + 2 * e + 1]);
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb) {
      x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(a + 16 * t * PITCH + cb * 64));
      x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(a + (16 * t + 8) * PITCH + cb * 64));
      if constexpr (SAFE) {
        Frag bad, one;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = (x.u[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (x.u[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
          x.u[e] &= ~(lo | hi);
          bad.u[e] = (lo | hi) & 0x3f803f80u;                     // 1 where the value is not finite
          one.u[e] = ((seen >> (8 * t + 2 * e)) & 1 ? 0x3f80u : 0u) | ((seen >> (8 * t + 2 * e + 1)) & 1 ? 0x3f800000u : 0u);
        }
        pk_f16 n{};
        n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bad.v, one.v, n, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (n[i] > 0.f) acc[cb][i] = __builtin_nanf("");
      }
      acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v, f.v, acc[cb], 0, 0, 0);
    }
  }
}
template <int D, bool SAFE>
__device__ __forceinline__ void pk_cols_f32(pk_f16 (&acc)[D / 32], const unsigned char* tile, int row0, const pk_f16& w, uint32_t seen,
                                            int lane) {
  constexpr int PITCH = PkTile<float, D>::PITCH;
  const unsigned char* a = tile + (row0 + 4 * (lane >> 5)) * PITCH + (lane & 31) * 4;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb) {
      float x = *reinterpret_cast<const float*>(a + (8 * (i >> 2) + (i & 3)) * PITCH + cb * 128);
      if constexpr (SAFE) {
        const bool bad = (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
        if (bad) x = 0.f;
        pk_f16 n{};
        n = __builtin_amdgcn_mfma_f32_32x32x2f32(bad ? 1.f : 0.f, (seen >> i) & 1 ? 1.f : 0.f, n, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (n[k] > 0.f) acc[cb][k] = __builtin_nanf("");
      }
      acc[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w[i], acc[cb], 0, 0, 0);
    }
  }
}
template <typename T, int D>
__device__ __forceinline__ void pk_product(pk_f16 (&acc)[D / 32], const unsigned char* tile, int row0, const pk_f16& w, bool safe,
                                           uint32_t seen, int lane) {
  if constexpr (sizeof(T) == 2) {
    if (safe) pk_cols<D, true>(acc, tile, row0, w, seen, lane);
    else pk_cols<D, false>(acc, tile, row0, w, seen, lane);
  } else {
    if (safe) pk_cols_f32<D, true>(acc, tile, row0, w, seen, lane);
    else pk_cols_f32<D, false>(acc, tile, row0, w, seen, lane);
  }
}

// ------------------------------------------------------------------ tiles
// Rows row0 .. row0 + 63 of a [row][D] matrix through registers into LDS; rows from `hi` on and columns from d on: zeros.
template <typename T, int D, bool VEC> struct PkStage {
  static constexpr int PPR = D * (int)sizeof(T) / 16, RP = 256 / PPR, N = PK_KT / RP, EPP = 16 / (int)sizeof(T);
  union Piece { uint4 u; T e[EPP]; };
  Piece v[N];
  __device__ __forceinline__ void load(const T* src, int64_t ld, int row0, int hi, int d) {
    const int r = threadIdx.x / PPR, c = (threadIdx.x % PPR) * EPP;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int row = row0 + r + RP * n;
      const T* p = src + (int64_t)row * ld + c;
      v[n].u = make_uint4(0, 0, 0, 0);
      if constexpr (VEC) {
        if (row < hi && c < d) v[n].u = *reinterpret_cast<const uint4*>(p);
      } else {
#pragma unroll
        for (int e = 0; e < EPP; ++e)
          if (row < hi && c + e < d) v[n].e[e] = p[e];
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char* tile) const {
    const int r = threadIdx.x / PPR, c = threadIdx.x % PPR;
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<uint4*>(tile + (r + RP * n) * PkTile<T, D>::PITCH + c * 16) = v[n].u;
  }
};

// a lane's row of a result: columns 32 cb + 8 (i/4) + 4 (l/32) + i%4
template <typename T, int D, bool VEC>
__device__ __forceinline__ void pk_store_row(T* row, const pk_f16 (&acc)[D / 32], float f, int d, int g) {
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = cb * 32 + q * 8 + 4 * g;
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

struct PkStr { int64_t b, r, h; };
struct PkArgs {
  const void *Q, *K, *V, *dCTX;
  const int32_t* off;
  void *CTX, *dQ, *dK, *dV;
  float *LSE, *Dsum;
  PkStr qs, ks, cs, dqs, dks;
  int B, R, nseq, Hq, Hkv, d, tiles, causal;
  float scale;
};

template <typename T> __device__ __forceinline__ const T* pk_at(const void* p, const PkStr& s, int b, int h) {
  return reinterpret_cast<const T*>(p) + b * s.b + h * s.h;
}
template <typename T> __device__ __forceinline__ T* pk_at(void* p, const PkStr& s, int b, int h) {
  return reinterpret_cast<T*>(p) + b * s.b + h * s.h;
}

// Workgroup -> (tile, key head, head of its group).  Key heads run fastest, so that where their number is a multiple of
// eight all workgroups that read one head's keys share an XCD's L2; the last tiles, which see the most keys, come first.
struct PkPlace {
  int b, hk, hq, t0;
  __device__ __forceinline__ PkPlace(const PkArgs& a, int group) {
    const int nk = a.B * a.Hkv, per = nk * group;
    const int tile = blockIdx.x / per, rest = blockIdx.x % per, kh = rest % nk;
    b = kh / a.Hkv;
    hk = kh % a.Hkv;
    hq = hk * (a.Hq / a.Hkv) + rest / nk;
    t0 = (a.tiles - 1 - tile) * PK_BM;
  }
};

// The rows of a workgroup: what each sees of the other side ([lo, hi), empty outside the sequences), what the workgroup
// and the wavefront see together, and what all rows of the wavefront see.
struct PkSpan {
  int row, lo, hi;
  bool in;
  int glo, ghi, wlo, whi, alo, ahi;
  // queries: keys from the sequence's start; keys: queries up to the sequence's end
  template <bool KEYS> __device__ __forceinline__ void init(PackedRows<PK_BM>& pr, int (&lim)[2], const PkArgs& a, int b, int t0) {
    pr.template scan<256>(a.off + (int64_t)b * (a.nseq + 1), a.nseq, a.R, t0);
    const int i = (threadIdx.x >> 6) * PK_WT + (threadIdx.x & 31);
    row = t0 + i;
    in = pr.range(t0, i, lo, hi);
    if (a.causal && in) {
      if (KEYS) lo = row;
      else hi = row + 1;
    }
    wlo = in ? lo : 0x7fffffff;
    whi = in ? hi : 0;
    alo = in ? lo : 0;
    ahi = in ? hi : 0x7fffffff;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
      wlo = min(wlo, __shfl_xor(wlo, s, 64));
      whi = max(whi, __shfl_xor(whi, s, 64));
      alo = max(alo, __shfl_xor(alo, s, 64));
      ahi = min(ahi, __shfl_xor(ahi, s, 64));
    }
    wlo = __builtin_amdgcn_readfirstlane(wlo);
    whi = __builtin_amdgcn_readfirstlane(whi);
    alo = __builtin_amdgcn_readfirstlane(alo);
    ahi = __builtin_amdgcn_readfirstlane(ahi);
    if (threadIdx.x == 0) { lim[0] = 0x7fffffff; lim[1] = 0; }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { atomicMin(&lim[0], wlo); atomicMax(&lim[1], whi); }
    __syncthreads();
    glo = __builtin_amdgcn_readfirstlane(lim[0]);
    ghi = __builtin_amdgcn_readfirstlane(lim[1]);
  }
  // bit i: row j0 + 8(i/4) + 4g + i%4 is among what this lane's row sees
  __device__ __forceinline__ uint32_t seen(int j0, int g) const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = j0 + 8 * (i >> 2) + 4 * g + (i & 3);
      m |= (j >= lo && j < hi ? 1u : 0u) << i;
    }
    return m;
  }
};

// ------------------------------------------------------------------ forward
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void pk_fwd_kernel(PkArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char sk[PkTile<T, D>::BYTES], sv[PkTile<T, D>::BYTES];
  __shared__ PackedRows<PK_BM> pr;
  __shared__ int lim[2];
  const int lane = threadIdx.x & 63, g = lane >> 5;
  const PkPlace at(a, a.Hq / a.Hkv);
  PkSpan sp;
  sp.template init<false>(pr, lim, a, at.b, at.t0);
  if (sp.glo >= sp.ghi) return;
  const T* kp = pk_at<T>(a.K, a.ks, at.b, at.hk);
  const T* vp = pk_at<T>(a.V, a.ks, at.b, at.hk);
  PkRow<T, D> q;
  pk_load_row<T, D, VEC>(q, pk_at<T>(a.Q, a.qs, at.b, at.hq) + (int64_t)sp.row * a.qs.r, sp.in, a.d, g);
  const float c = a.scale * PK_LOG2E;
  for (bool safe = false;; safe = true) {
    pk_f16 o[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = pk_f16{};
    float m = -INFINITY, l = 0.f;
    PkStage<T, D, VEC> nk, nv;
    nk.load(kp, a.ks.r, sp.glo, sp.ghi, a.d);
    nv.load(vp, a.ks.r, sp.glo, sp.ghi, a.d);
    for (int k0 = sp.glo; k0 < sp.ghi; k0 += PK_KT) {
      __syncthreads();
      nk.store(sk);
      nv.store(sv);
      __syncthreads();
      if (k0 + PK_KT < sp.ghi) {
        nk.load(kp, a.ks.r, k0 + PK_KT, sp.ghi, a.d);
        nv.load(vp, a.ks.r, k0 + PK_KT, sp.ghi, a.d);
      }
      if (k0 >= sp.whi || k0 + PK_KT <= sp.wlo) continue;
      pk_f16 s[2] = {pk_f16{}, pk_f16{}};
      float mt = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        pk_rows<D>(s[kb], sk, kb * 32, q, lane);
        if (k0 < sp.alo || k0 + PK_KT > sp.ahi) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = k0 + kb * 32 + 8 * (i >> 2) + 4 * g + (i & 3);
            if (j < sp.lo || j >= sp.hi) s[kb][i] = -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[kb][i]);
      }
      mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
      const float mn = fmaxf(m, c * mt), mu = mn == -INFINITY ? 0.f : mn;
      if (__any(mn > m)) {
        const float f = pk_exp2(m - mu);
        l *= f;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[n][i] *= f;
        m = mn;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kb][i] = pk_exp2(fmaf(c, s[kb][i], -mu));
          l += s[kb][i];
        }
        pk_product<T, D>(o, sv, kb * 32, s[kb], safe, safe ? sp.seen(k0 + kb * 32, g) : 0u, lane);
      }
    }
    if (!safe && __syncthreads_or(sp.in && pk_not_finite(o))) continue;
    l += __shfl_xor(l, 32, 64);
    if (sp.in) {
      pk_store_row<T, D, VEC>(pk_at<T>(a.CTX, a.cs, at.b, at.hq) + (int64_t)sp.row * a.cs.r, o, 1.f / l, a.d, g);
      if (g == 0) a.LSE[((int64_t)at.b * a.Hq + at.hq) * a.R + sp.row] = (m + __builtin_amdgcn_logf(l)) * PK_LN2;
    }
    return;
  }
}

// ------------------------------------------------------------------ backward: D and dQ
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void pk_dq_kernel(PkArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char sk[PkTile<T, D>::BYTES], sv[PkTile<T, D>::BYTES];
  __shared__ PackedRows<PK_BM> pr;
  __shared__ int lim[2];
  const int lane = threadIdx.x & 63, g = lane >> 5;
  const PkPlace at(a, a.Hq / a.Hkv);
  PkSpan sp;
  sp.template init<false>(pr, lim, a, at.b, at.t0);
  if (sp.glo >= sp.ghi) return;
  const T* kp = pk_at<T>(a.K, a.ks, at.b, at.hk);
  const T* vp = pk_at<T>(a.V, a.ks, at.b, at.hk);
  const int64_t srow = ((int64_t)at.b * a.Hq + at.hq) * a.R + sp.row;
  PkRow<T, D> q, dc;
  pk_load_row<T, D, VEC>(q, pk_at<T>(a.Q, a.qs, at.b, at.hq) + (int64_t)sp.row * a.qs.r, sp.in, a.d, g);
  pk_load_row<T, D, VEC>(dc, pk_at<T>(a.dCTX, a.cs, at.b, at.hq) + (int64_t)sp.row * a.cs.r, sp.in, a.d, g);
  float dsum = 0.f;
  {
    PkRow<T, D> x;
    pk_load_row<T, D, VEC>(x, pk_at<T>(a.CTX, a.cs, at.b, at.hq) + (int64_t)sp.row * a.cs.r, sp.in, a.d, g);
#pragma unroll
    for (int s = 0; s < PkRow<T, D>::N; ++s)
#pragma unroll
      for (int e = 0; e < PkRow<T, D>::EPP; ++e) dsum = fmaf(Elem<T>::to_f32(x.p[s].e[e]), Elem<T>::to_f32(dc.p[s].e[e]), dsum);
    dsum += __shfl_xor(dsum, 32, 64);
  }
  const float lse = sp.in ? a.LSE[srow] * PK_LOG2E : 0.f;
  if (sp.in && g == 0) a.Dsum[srow] = dsum;
  const float c = a.scale * PK_LOG2E;
  for (bool safe = false;; safe = true) {
    pk_f16 o[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = pk_f16{};
    PkStage<T, D, VEC> nk, nv;
    nk.load(kp, a.ks.r, sp.glo, sp.ghi, a.d);
    nv.load(vp, a.ks.r, sp.glo, sp.ghi, a.d);
    for (int k0 = sp.glo; k0 < sp.ghi; k0 += PK_KT) {
      __syncthreads();
      nk.store(sk);
      nv.store(sv);
      __syncthreads();
      if (k0 + PK_KT < sp.ghi) {
        nk.load(kp, a.ks.r, k0 + PK_KT, sp.ghi, a.d);
        nv.load(vp, a.ks.r, k0 + PK_KT, sp.ghi, a.d);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int j0 = k0 + kb * 32;
        if (j0 >= sp.whi || j0 + 32 <= sp.wlo) continue;
        pk_f16 s{}, p{};
        pk_rows<D>(s, sk, kb * 32, q, lane);
        pk_rows<D>(p, sv, kb * 32, dc, lane);
        const uint32_t seen = j0 < sp.alo || j0 + 32 > sp.ahi || safe ? sp.seen(j0, g) : 0xffffu;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = pk_exp2(fmaf(c, s[i], -lse)) * (p[i] - dsum);
          s[i] = (seen >> i) & 1 ? x : 0.f;
        }
        pk_product<T, D>(o, sk, kb * 32, s, safe, seen, lane);
      }
    }
    if (!safe && __syncthreads_or(sp.in && pk_not_finite(o))) continue;
    if (sp.in) pk_store_row<T, D, VEC>(pk_at<T>(a.dQ, a.dqs, at.b, at.hq) + (int64_t)sp.row * a.dqs.r, o, a.scale, a.d, g);
    return;
  }
}

// ------------------------------------------------------------------ backward: dK and dV
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void pk_dkv_kernel(PkArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char sq[PkTile<T, D>::BYTES], sc[PkTile<T, D>::BYTES];
  __shared__ __attribute__((aligned(16))) float sl[PK_KT], sd[PK_KT];
  __shared__ PackedRows<PK_BM> pr;
  __shared__ int lim[2];
  const int lane = threadIdx.x & 63, g = lane >> 5;
  const PkPlace at(a, 1);
  PkSpan sp;
  sp.template init<true>(pr, lim, a, at.b, at.t0);
  if (sp.glo >= sp.ghi) return;
  const int group = a.Hq / a.Hkv;
  PkRow<T, D> k, v;
  pk_load_row<T, D, VEC>(k, pk_at<T>(a.K, a.ks, at.b, at.hk) + (int64_t)sp.row * a.ks.r, sp.in, a.d, g);
  pk_load_row<T, D, VEC>(v, pk_at<T>(a.V, a.ks, at.b, at.hk) + (int64_t)sp.row * a.ks.r, sp.in, a.d, g);
  const float c = a.scale * PK_LOG2E;
  for (bool safe = false;; safe = true) {
    pk_f16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = pk_f16{};
    for (int h = at.hq; h < at.hq + group; ++h) {
      const T* qp = pk_at<T>(a.Q, a.qs, at.b, h);
      const T* cp = pk_at<T>(a.dCTX, a.cs, at.b, h);
      const float* lp = a.LSE + ((int64_t)at.b * a.Hq + h) * a.R;
      const float* dp = a.Dsum + ((int64_t)at.b * a.Hq + h) * a.R;
      PkStage<T, D, VEC> nq, nc;
      float nl = 0.f;
      auto fetch = [&](int i0) {
        nq.load(qp, a.qs.r, i0, sp.ghi, a.d);
        nc.load(cp, a.cs.r, i0, sp.ghi, a.d);
        if (threadIdx.x < 2 * PK_KT) {
          const int i = i0 + (threadIdx.x & 63);
          nl = i < sp.ghi ? (threadIdx.x < PK_KT ? lp[i] * PK_LOG2E : dp[i]) : 0.f;
        }
      };
      fetch(sp.glo);
      for (int i0 = sp.glo; i0 < sp.ghi; i0 += PK_KT) {
        __syncthreads();
        nq.store(sq);
        nc.store(sc);
        if (threadIdx.x < 2 * PK_KT) (threadIdx.x < PK_KT ? sl : sd)[threadIdx.x & 63] = nl;
        __syncthreads();
        if (i0 + PK_KT < sp.ghi) fetch(i0 + PK_KT);
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
          const int j0 = i0 + qb * 32;
          if (j0 >= sp.whi || j0 + 32 <= sp.wlo) continue;
          pk_f16 s{}, p{};
          pk_rows<D>(s, sq, qb * 32, k, lane);
          pk_rows<D>(p, sc, qb * 32, v, lane);
          const uint32_t seen = j0 < sp.alo || j0 + 32 > sp.ahi || safe ? sp.seen(j0, g) : 0xffffu;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float4 ls = *reinterpret_cast<const float4*>(sl + qb * 32 + n * 8 + 4 * g);
            const float4 ds = *reinterpret_cast<const float4*>(sd + qb * 32 + n * 8 + 4 * g);
            const float lv[4] = {ls.x, ls.y, ls.z, ls.w}, dd[4] = {ds.x, ds.y, ds.z, ds.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = 4 * n + e;
              const float x = pk_exp2(fmaf(c, s[i], -lv[e]));
              const bool ok = (seen >> i) & 1;
              s[i] = ok ? x : 0.f;
              p[i] = ok ? x * (p[i] - dd[e]) : 0.f;
            }
          }
          pk_product<T, D>(dv, sc, qb * 32, s, safe, seen, lane);
          pk_product<T, D>(dk, sq, qb * 32, p, safe, seen, lane);
        }
      }
    }
    if (!safe && __syncthreads_or(sp.in && (pk_not_finite(dk) || pk_not_finite(dv)))) continue;
    if (sp.in) {
      pk_store_row<T, D, VEC>(pk_at<T>(a.dK, a.dks, at.b, at.hk) + (int64_t)sp.row * a.dks.r, dk, a.scale, a.d, g);
      pk_store_row<T, D, VEC>(pk_at<T>(a.dV, a.dks, at.b, at.hk) + (int64_t)sp.row * a.dks.r, dv, 1.f, a.d, g);
    }
    return;
  }
}

// ------------------------------------------------------------------ host side
int pk_check(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, float scale) {
  if (B <= 0 || R <= 0 || nseq <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv || !valid_dtype(dtype) || !(scale > 0.f) ||
      isinf(scale) || R > 0x7fffffff - PK_BM)
    return HFTA_EINVAL;
  const int64_t tiles = (R + PK_BM - 1) / PK_BM;
  return d > 128 || (int64_t)B * Hq > 0x7fffffff / tiles ? HFTA_EUNSUPPORTED : HFTA_OK;
}
PkStr pk_str(const int64_t* s) { return s ? PkStr{s[0], s[1], s[2]} : PkStr{0, 0, 0}; }

// rows in whole 16-byte pieces: pointers, strides and head widths
bool pk_pieces(const PkArgs& a, int dtype, const void* const* p, int n) {
  const int64_t m = dtype == HFTA_BF16 ? 8 : 4;
  uintptr_t bits = 0;
  for (int i = 0; i < n; ++i) bits |= reinterpret_cast<uintptr_t>(p[i]);
  const PkStr* s[] = {&a.qs, &a.ks, &a.cs, &a.dqs, &a.dks};
  for (const PkStr* x : s)
    if (x->b % m || x->r % m || x->h % m) return false;
  return a.d % m == 0 && bits % 16 == 0;
}

#define PK_LAUNCH(KERNEL, GRID)                                                                              \
  do {                                                                                                       \
    const dim3 grid_(GRID), block_(256);                                                                     \
    if (dtype == HFTA_BF16) {                                                                                \
      if (a.d <= 32) vec ? KERNEL<bf16_raw, 32, true><<<grid_, block_, 0, st>>>(a) : KERNEL<bf16_raw, 32, false><<<grid_, block_, 0, st>>>(a);   \
      else if (a.d <= 64) vec ? KERNEL<bf16_raw, 64, true><<<grid_, block_, 0, st>>>(a) : KERNEL<bf16_raw, 64, false><<<grid_, block_, 0, st>>>(a); \
      else vec ? KERNEL<bf16_raw, 128, true><<<grid_, block_, 0, st>>>(a) : KERNEL<bf16_raw, 128, false><<<grid_, block_, 0, st>>>(a);           \
    } else {                                                                                                 \
      if (a.d <= 32) vec ? KERNEL<float, 32, true><<<grid_, block_, 0, st>>>(a) : KERNEL<float, 32, false><<<grid_, block_, 0, st>>>(a);         \
      else if (a.d <= 64) vec ? KERNEL<float, 64, true><<<grid_, block_, 0, st>>>(a) : KERNEL<float, 64, false><<<grid_, block_, 0, st>>>(a);    \
      else vec ? KERNEL<float, 128, true><<<grid_, block_, 0, st>>>(a) : KERNEL<float, 128, false><<<grid_, block_, 0, st>>>(a);                 \
    }                                                                                                        \
  } while (0)

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" {

int hfta_attention_packed_fwd(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3],
                              const void* K, const void* V, const int64_t kvs[3], const int32_t* seq_offsets, float scale,
                              int causal, void* CTX, const int64_t cs[3], float* LSE, void* stream) {
  const int rc = pk_check(B, R, nseq, Hq, Hkv, d, dtype, scale);
  if (rc == HFTA_EINVAL || !Q || !qs || !K || !V || !kvs || !seq_offsets || !CTX || !cs || !LSE) return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  PkArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.off = seq_offsets; a.CTX = CTX; a.LSE = LSE;
  a.qs = pk_str(qs); a.ks = pk_str(kvs); a.cs = pk_str(cs);
  a.B = B; a.R = R; a.nseq = nseq; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.causal = causal != 0; a.scale = scale;
  a.tiles = (R + PK_BM - 1) / PK_BM;
  const void* p[] = {Q, K, V, CTX};
  const bool vec = pk_pieces(a, dtype, p, 4);
  hipStream_t st = as_stream(stream);
  PK_LAUNCH(pk_fwd_kernel, (unsigned)(a.tiles * B * Hq));
  return launch_status();
}

size_t hfta_attention_packed_bwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  if (pk_check(B, R, nseq, Hq, Hkv, d, dtype, 1.f) != HFTA_OK) return 0;
  return (size_t)B * Hq * R * sizeof(float);
}

int hfta_attention_packed_bwd(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3],
                              const void* K, const void* V, const int64_t kvs[3], const int32_t* seq_offsets, float scale,
                              int causal, const void* CTX, const void* dCTX, const int64_t cs[3], const float* LSE,
                              void* dQ, const int64_t dqs[3], void* dK, void* dV, const int64_t dkvs[3],
                              void* workspace, size_t ws_bytes, void* stream) {
  const int rc = pk_check(B, R, nseq, Hq, Hkv, d, dtype, scale);
  if (rc == HFTA_EINVAL || !Q || !qs || !K || !V || !kvs || !seq_offsets || !CTX || !dCTX || !cs || !LSE || !dQ || !dqs || !dK ||
      !dV || !dkvs)
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 4 ||
      ws_bytes < hfta_attention_packed_bwd_workspace_bytes(B, R, nseq, Hq, Hkv, d, dtype))
    return HFTA_EWORKSPACE;
  PkArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.dCTX = dCTX; a.off = seq_offsets; a.CTX = const_cast<void*>(CTX); a.LSE = const_cast<float*>(LSE);
  a.dQ = dQ; a.dK = dK; a.dV = dV; a.Dsum = reinterpret_cast<float*>(workspace);
  a.qs = pk_str(qs); a.ks = pk_str(kvs); a.cs = pk_str(cs); a.dqs = pk_str(dqs); a.dks = pk_str(dkvs);
  a.B = B; a.R = R; a.nseq = nseq; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.causal = causal != 0; a.scale = scale;
  a.tiles = (R + PK_BM - 1) / PK_BM;
  const void* p[] = {Q, K, V, CTX, dCTX, dQ, dK, dV};
  const bool vec = pk_pieces(a, dtype, p, 8);
  hipStream_t st = as_stream(stream);
  PK_LAUNCH(pk_dq_kernel, (unsigned)(a.tiles * B * Hq));
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  PK_LAUNCH(pk_dkv_kernel, (unsigned)(a.tiles * B * Hkv));
  return launch_status();
}

}  // extern "C"
