// What stands between two blocks of a decoder layer, in one call per direction (fusion rules table rows "LayerNorm" and element-wise):
// the block's own norm, its gate and residual scale, the sum with the residual stream and the norm in front of the next block.
//
//   u = N(F) w1 + b1,   S = X + res sigma(G) u,   Y = N(S) w2 + b2
//   N(z) = (z - mean z) / sqrt(var z + eps),  or  z / sqrt(mean z^2 + eps)  (RMS)
//
// and backwards, with sh = N(S), fh = N(F), h = sigma(G), and t of a norm with inverse deviation i: N'(t, zh, i) = i (t - mean t - zh mean(t zh)):
//   ds = dS + N'(dY w2, sh, i2),   dX = ds,   du = res h ds,   dF = N'(du w1, fh, i1),   dG = res ds u h (1 - h)
//   dw1 = sum du fh,  db1 = sum du,  dw2 = sum dY sh,  db2 = sum dY,  dres = sum h u ds      (sums over rows)
//
// Bound by memory: a row is read once and stays in registers, a thread's share of 8 elements (16 past 8192 columns), through both norms; a row has as many
// threads as that takes: 8 or 32 lanes, a wavefront, 128 to 1024 threads.  5 x 9633 rows, bf16, both directions: 30 us at 16 columns and 76 at 200, where
// a wavefront for each row took 125 and 132; 32 lanes for 16 columns would leave three quarters of them idle.  The backward call forms S
// again from X, F and G rather than read its rounded copy (as many bytes, and the gradients are those of what Y was made of).  Sums over rows stay in
// registers across a workgroup's rows, pass through the workspace and are added in order.
//
// 2 x 8192 rows of 2048 bf16, gate, without means: forward 77 us (10 bytes an element, 4.4 TB/s), backward 130 (16 bytes, 4.1 TB/s), sums 15.
#include "pieces.h"

#include <type_traits>

namespace hfta {
namespace {

struct GnArgs {
  const void *X, *F, *G, *dS, *dY;
  const float *w1, *b1, *res, *w2, *b2;
  void *S, *Y, *dX, *dF, *dG;
  float *m1, *i1, *m2, *i2, *part;
  float eps;
  int R, E, blocks;                // blocks: workgroups of a model
};
constexpr int GN_MAX_BLOCKS = 1024;
constexpr int gn_threads(int tpr) { return tpr < 256 && tpr != 128 ? 256 : tpr; }      // of a workgroup, by the threads of a row

template <int TPR> struct GnSum {
  float lds[2][2][TPR > 64 ? TPR / 64 : 1];
};
// the sum over a row's lanes of a wavefront
template <int TPR> __device__ __forceinline__ float gn_lanes(float x) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
// two sums over the TPR threads of a row; `turn` alternates between calls, so that one barrier is enough
template <int TPR> __device__ __forceinline__ void gn_sum(GnSum<TPR>& s, int turn, float& x, float& y) {
  x = gn_lanes<TPR>(x);
  y = gn_lanes<TPR>(y);
  if constexpr (TPR > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { s.lds[turn][0][w] = x; s.lds[turn][1][w] = y; }
    __syncthreads();
    x = y = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) { x += s.lds[turn][0][i]; y += s.lds[turn][1][i]; }
  }
}

// a thread's share of a row: NP pieces, TPR pieces apart
template <typename T, int NP, int TPR> struct GnRow {
  typedef Piece16<T> P;
  static constexpr int N = NP * P::N;
  static __device__ __forceinline__ int col(int p) { return (p * TPR + (int)(threadIdx.x % TPR)) * P::N; }
  static __device__ __forceinline__ void load(float (&x)[NP][P::N], const T* row, int E) {
#pragma unroll
    for (int p = 0; p < NP; ++p) P::load(x[p], row + col(p), E - col(p));
  }
  static __device__ __forceinline__ void store(T* row, const float (&x)[NP][P::N], int E) {
#pragma unroll
    for (int p = 0; p < NP; ++p) P::store(row + col(p), x[p], E - col(p));
  }
  // fp32 rows of weights (NULL: `none`)
  static __device__ __forceinline__ void weights(float (&x)[NP][P::N], const float* row, int E, float none) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if (!row) {
#pragma unroll
        for (int e = 0; e < P::N; ++e) x[p][e] = none;
        continue;
      }
#pragma unroll
      for (int q = 0; q < P::N / 4; ++q) {
        float w[4];
        Piece16<float>::load(w, row + col(p) + 4 * q, E - col(p) - 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[p][4 * q + e] = w[e];
      }
    }
  }
};
#define GN_EACH(NP, N)                 \
  _Pragma("unroll") for (int p = 0; p < NP; ++p) _Pragma("unroll") for (int e = 0; e < N; ++e)

// the statistics of a row; x becomes x - mean where means are taken (zeros behind the row stay zeros)
template <typename T, int NP, int TPR, bool RMS>
__device__ __forceinline__ void gn_stats(GnSum<TPR>& sum, int& turn, float (&x)[NP][Piece16<T>::N], int E, float eps, float& mean, float& inv) {
  typedef GnRow<T, NP, TPR> Row;
  constexpr int N = Piece16<T>::N;
  float s = 0.f, z = 0.f;
  mean = 0.f;
  if constexpr (!RMS) {
    GN_EACH(NP, N) s += x[p][e];
    gn_sum<TPR>(sum, turn, s, z);
    turn ^= 1;
    mean = s / (float)E;
    GN_EACH(NP, N) x[p][e] = Row::col(p) + e < E ? x[p][e] - mean : 0.f;
  }
  s = z = 0.f;
  GN_EACH(NP, N) s = fmaf(x[p][e], x[p][e], s);
  gn_sum<TPR>(sum, turn, s, z);
  turn ^= 1;
  inv = 1.f / sqrtf(s / (float)E + eps);
}

__device__ __forceinline__ float gn_sigma(float x) { return 1.f / (1.f + expf(-x)); }
// A gate h = sigma(x) and 1 - h, each with its own digits (1 - h of an open gate, subtracted from one, has none left past x = 17)
struct GnTwo {
  float h, shut;
  __device__ __forceinline__ void set(float x) {
    const float e = expf(-x);
    h = 1.f / (1.f + e);
    shut = x > 0.f ? e * h : 1.f - h;
  }
  __device__ __forceinline__ void none() { h = 1.f; }
  __device__ __forceinline__ float open() const { return h; }
  __device__ __forceinline__ float closed() const { return shut; }
};
// the same in one register: the smaller of the two, 1 - h with its sign set
struct GnOne {
  float v;
  __device__ __forceinline__ void set(float x) {
    const float e = expf(-fabsf(x)), y = 1.f / (1.f + e);
    v = copysignf(e * y, -x);
  }
  __device__ __forceinline__ void none() { v = 1.f; }
  __device__ __forceinline__ int side() const { return __float_as_int(v) >> 31; }
  __device__ __forceinline__ float open() const { return __int_as_float(side() & 0x3f800000) + v; }
  __device__ __forceinline__ float closed() const { return __int_as_float(~side() & 0x3f800000) - v; }
};

template <typename T, int NP, int TPR, bool RMS, bool BLOCK>
__global__ __launch_bounds__(gn_threads(TPR)) void gn_fwd_kernel(GnArgs a) {
  typedef GnRow<T, NP, TPR> Row;
  constexpr int N = Piece16<T>::N, NT = gn_threads(TPR), RPB = NT / TPR;
  __shared__ GnSum<TPR> sum;
  const int b = blockIdx.y, E = a.E;
  const int r = blockIdx.x * RPB + threadIdx.x / TPR;
  if (r >= a.R) return;                                          // (all lanes of a row; workgroups of one row never)
  const int64_t row = (int64_t)b * a.R + r, at = row * E;
  int turn = 0;
  float f[NP][N], x[NP][N];
  Row::load(x, reinterpret_cast<const T*>(a.X) + at, E);
  if constexpr (BLOCK) {
    Row::load(f, reinterpret_cast<const T*>(a.F) + at, E);
    float w[NP][N], c[NP][N], mean, inv;
    Row::weights(w, a.w1 + (int64_t)b * E, E, 0.f);
    Row::weights(c, a.b1 ? a.b1 + (int64_t)b * E : nullptr, E, 0.f);
    const float res = a.res ? a.res[b] : 1.f;
    float g[NP][N];
    if (a.G) Row::load(g, reinterpret_cast<const T*>(a.G) + at, E);
    gn_stats<T, NP, TPR, RMS>(sum, turn, f, E, a.eps, mean, inv);
    if (threadIdx.x % TPR == 0) {
      if (!RMS) a.m1[row] = mean;
      a.i1[row] = inv;
    }
    GN_EACH(NP, N) {
      const float h = a.G ? res * gn_sigma(g[p][e]) : res;
      if (Row::col(p) + e < E) x[p][e] = fmaf(h, fmaf(f[p][e] * inv, w[p][e], c[p][e]), x[p][e]);
    }
    Row::store(reinterpret_cast<T*>(a.S) + at, x, E);
  }
  float w[NP][N], c[NP][N], mean, inv;
  Row::weights(w, a.w2 + (int64_t)b * E, E, 0.f);
  Row::weights(c, a.b2 ? a.b2 + (int64_t)b * E : nullptr, E, 0.f);
  gn_stats<T, NP, TPR, RMS>(sum, turn, x, E, a.eps, mean, inv);
  if (threadIdx.x % TPR == 0) {
    if (!RMS) a.m2[row] = mean;
    a.i2[row] = inv;
  }
  GN_EACH(NP, N) x[p][e] = fmaf(x[p][e] * inv, w[p][e], c[p][e]);
  Row::store(reinterpret_cast<T*>(a.Y) + at, x, E);
}

// Partial sums of a workgroup's rows, in part[model][workgroup][4 E + 4] (dw2, db2, dw1, db1, and dres in the next word).  The next row is on its way
// while one is computed (the case above: 227 -> 130 us; with four wavefronts a SIMD instead of three its registers spill).  1024 threads leave a thread
// 128 registers, too few to hold a second row, and with the block's norm too few for one: from 4097 columns on 40 to 160 bytes of a thread pass through
// scratch memory, past 8192 500 to 780.  BIAS: sums of the gradients themselves are wanted; without them (a norm without biases) 16 registers are free.
template <typename T, int NP, int TPR, bool RMS, bool BLOCK, bool BIAS>
__global__ __launch_bounds__(gn_threads(TPR), (TPR == 1024 ? 4 : BIAS || sizeof(T) == 4 || TPR == 512 ? 2 : 3)) void gn_bwd_kernel(GnArgs a) {
  typedef GnRow<T, NP, TPR> Row;
  typedef Piece16<T> P;
  constexpr int N = P::N, NT = gn_threads(TPR), RPB = NT / TPR;
  constexpr bool AHEAD = TPR < 1024;
  // Registers for 1 - h: without biases, and with the few of 1024 threads, u is formed again rather than held, past 8192 columns from biases loaded again,
  // and with 1024 threads a gate is one register (2 x 2048 rows of 8192 bf16, both directions: 279 us, with two 303; 5 x 9633 rows of 200, means
  // and biases: 99 and 95)
  constexpr bool AGAIN = TPR == 1024 || !BIAS, LOADS = BIAS && NP * N > 8;
  typedef std::conditional_t<TPR == 1024, GnOne, GnTwo> Gate;
  __shared__ GnSum<TPR> sum;
  const int b = blockIdx.y, E = a.E;
  const float res = BLOCK && a.res ? a.res[b] : 1.f;
  const float *w1 = a.w1 + (int64_t)b * E, *b1 = a.b1 ? a.b1 + (int64_t)b * E : nullptr, *w2 = a.w2 + (int64_t)b * E;
  float dw1[NP][N], db1[NP][N], dw2[NP][N], db2[NP][N], dres = 0.f;
  GN_EACH(NP, N) dw1[p][e] = db1[p][e] = dw2[p][e] = db2[p][e] = 0.f;
  int first = blockIdx.x * RPB + threadIdx.x / TPR;
  if (TPR >= 64) first = __builtin_amdgcn_readfirstlane(first);
  const int step = a.blocks * RPB;
  float w[NP][N], c[NP][N], v[NP][N];
  auto weights = [&]() __attribute__((always_inline)) {
    if constexpr (BLOCK) {
      Row::weights(w, w1, E, 0.f);
      if (BIAS) Row::weights(c, b1, E, 0.f);
    }
    Row::weights(v, w2, E, 0.f);
  };
  struct Raw { piece_u4 x[NP], f[NP], g[NP], dy[NP], ds[NP]; } in;
  float m1 = 0.f, i1 = 0.f, m2 = 0.f, i2;
  auto load = [&](int r) __attribute__((always_inline)) {
    const int64_t row = (int64_t)b * a.R + r, at = row * E;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int col = Row::col(p), n = E - col;
      const int64_t to = at + col;
      in.x[p] = P::raw(reinterpret_cast<const T*>(a.X) + to, n);
      if constexpr (BLOCK) {
        in.f[p] = P::raw(reinterpret_cast<const T*>(a.F) + to, n);
        if (a.G) in.g[p] = P::raw(reinterpret_cast<const T*>(a.G) + to, n);
      }
      in.dy[p] = P::raw(reinterpret_cast<const T*>(a.dY) + to, n);
      if (a.dS) in.ds[p] = P::raw(reinterpret_cast<const T*>(a.dS) + to, n);
    }
    i2 = a.i2[row];
    if (!RMS) m2 = a.m2[row];
    if constexpr (BLOCK) {
      i1 = a.i1[row];
      if (!RMS) m1 = a.m1[row];
    }
  };
  int turn = 0;
  if (AHEAD && first < a.R) load(first);
  for (int r = first; r < a.R; r += step) {
    const int64_t at = ((int64_t)b * a.R + r) * E;
    if (!AHEAD) load(r);
    float x[NP][N], f[NP][N], gx[NP][N], dy[NP][N], ds[NP][N];
    Gate g[NP][N];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      P::values(x[p], in.x[p]);
      if constexpr (BLOCK) {
        P::values(f[p], in.f[p]);
        if constexpr (AHEAD) {                                    // (gates are formed with the next row's loads on their way)
          if (a.G) P::values(gx[p], in.g[p]);
        } else if (a.G) {
          float raw[N];
          P::values(raw, in.g[p]);
#pragma unroll
          for (int e = 0; e < N; ++e) g[p][e].set(raw[e]);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) g[p][e].none();
        }
      }
      P::values(dy[p], in.dy[p]);
      if (a.dS) P::values(ds[p], in.ds[p]);
    }
    auto block = [&](int p, int e) __attribute__((always_inline)) { return BIAS ? fmaf(f[p][e], w[p][e], c[p][e]) : f[p][e] * w[p][e]; };     // u
    const float mean1 = m1, inv1 = i1, mean2 = m2, inv2 = i2;
    if (AHEAD && r + step < a.R) load(r + step);
    weights();
    if constexpr (BLOCK) {
      GN_EACH(NP, N) {
        f[p][e] = RMS ? f[p][e] * inv1 : Row::col(p) + e < E ? (f[p][e] - mean1) * inv1 : 0.f;
        if constexpr (AHEAD) {
          if (a.G) g[p][e].set(gx[p][e]);
          else g[p][e].none();
        }
        x[p][e] = fmaf(res * g[p][e].open(), block(p, e), x[p][e]);
      }
    }
    float s = 0.f, z = 0.f;
    GN_EACH(NP, N) {
      x[p][e] = RMS ? x[p][e] * inv2 : Row::col(p) + e < E ? (x[p][e] - mean2) * inv2 : 0.f;
      dw2[p][e] = fmaf(dy[p][e], x[p][e], dw2[p][e]);
      if (BIAS) db2[p][e] += dy[p][e];
      dy[p][e] *= v[p][e];
      s = fmaf(dy[p][e], x[p][e], s);
      if (!RMS) z += dy[p][e];
    }
    gn_sum<TPR>(sum, turn, s, z);
    turn ^= 1;
    s /= (float)E;
    z /= (float)E;
    GN_EACH(NP, N) ds[p][e] = inv2 * (dy[p][e] - z - x[p][e] * s) + (a.dS ? ds[p][e] : 0.f);
    Row::store(reinterpret_cast<T*>(a.dX) + at, ds, E);
    if constexpr (BLOCK) {
      s = z = 0.f;
      if constexpr (LOADS) Row::weights(c, b1, E, 0.f);
      if constexpr (AGAIN) {
        GN_EACH(NP, N) asm volatile("" : "+v"(f[p][e]));
      }
      GN_EACH(NP, N) {
        const float u = block(p, e);
        const float hd = RMS || Row::col(p) + e < E ? g[p][e].open() * ds[p][e] : 0.f, du = res * hd;       // (z makes ds not zero behind the row)
        dres = fmaf(hd, u, dres);
        dw1[p][e] = fmaf(du, f[p][e], dw1[p][e]);
        if (BIAS) db1[p][e] += du;
        ds[p][e] = du * u * g[p][e].closed();                     // dG
        dy[p][e] = du * w[p][e];
        s = fmaf(dy[p][e], f[p][e], s);
        if (!RMS) z += dy[p][e];
      }
      if (a.G) Row::store(reinterpret_cast<T*>(a.dG) + at, ds, E);
      gn_sum<TPR>(sum, turn, s, z);
      turn ^= 1;
      s /= (float)E;
      z /= (float)E;
      GN_EACH(NP, N) dy[p][e] = inv1 * (dy[p][e] - z - f[p][e] * s);
      Row::store(reinterpret_cast<T*>(a.dF) + at, dy, E);
    }
  }
  if constexpr (TPR < 64) {                                      // a wavefront's rows
    auto rows = [](float& x) __attribute__((always_inline)) {
#pragma unroll
      for (int o = TPR; o < 64; o <<= 1) x += __shfl_xor(x, o, 64);
    };
    GN_EACH(NP, N) {
      rows(dw2[p][e]);
      if (BIAS) rows(db2[p][e]);
      if (BLOCK) rows(dw1[p][e]);
      if (BLOCK && BIAS) rows(db1[p][e]);
    }
    if (BLOCK) rows(dres);
  }
  float* out = a.part + ((int64_t)b * a.blocks + blockIdx.x) * (4 * (int64_t)E + 4);
  if constexpr (TPR <= 64) {                                     // and a workgroup's
    constexpr int WAVES = NT / 64;
    __shared__ float lds[WAVES][TPR * NP * N];
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
    auto put = [&](float* to, const float (&y)[NP][N]) __attribute__((always_inline)) {
      __syncthreads();
      if (lane < TPR) {
        GN_EACH(NP, N) lds[wv][Row::col(p) + e] = y[p][e];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < E; c += NT) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += lds[w][c];
        to[c] = x;
      }
    };
    put(out, dw2);
    if (BIAS) put(out + E, db2);
    if constexpr (BLOCK) {
      put(out + 2 * (int64_t)E, dw1);
      if (BIAS) put(out + 3 * (int64_t)E, db1);
      dres = gn_lanes<TPR>(dres);
      __syncthreads();
      if (lane == 0) lds[wv][0] = dres;
      __syncthreads();
      if (threadIdx.x == 0) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += lds[w][0];
        out[4 * (int64_t)E] = x;
      }
    }
  } else {
    auto put = [&](float* to, const float (&y)[NP][N]) __attribute__((always_inline)) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
          const float w4[4] = {y[p][4 * q], y[p][4 * q + 1], y[p][4 * q + 2], y[p][4 * q + 3]};
          Piece16<float>::store(to + Row::col(p) + 4 * q, w4, E - Row::col(p) - 4 * q);
        }
    };
    put(out, dw2);
    if (BIAS) put(out + E, db2);
    if constexpr (BLOCK) {
      put(out + 2 * (int64_t)E, dw1);
      if (BIAS) put(out + 3 * (int64_t)E, db1);
      float none = 0.f;
      gn_sum<TPR>(sum, turn, dres, none);
      if (threadIdx.x == 0) out[4 * (int64_t)E] = dres;
    }
  }
}

// The parts of a model added in order: a workgroup takes 64 columns, each of its wavefronts a sixteenth of the parts, sixteen in flight
constexpr int GN_ADD = 1024;
__global__ __launch_bounds__(GN_ADD) void gn_add_kernel(const float* part, int parts, int E, float* dw2, float* db2, float* dw1, float* db1, float* dres) {
  constexpr int W = GN_ADD / 64, AHEAD = 16;
  __shared__ double lds[W][64];
  const int b = blockIdx.y, q = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t width = 4 * (int64_t)E + 4, c = (int64_t)blockIdx.x * 64 + lane;
  const int which = c < 4 * (int64_t)E ? (int)(c / E) : 4;
  float* out = which == 0 ? dw2 : which == 1 ? db2 : which == 2 ? dw1 : which == 3 ? db1 : dres;
  const bool has = out && c <= 4 * (int64_t)E;
  if (!__syncthreads_or(has)) return;                            // (sums that nobody asked for)
  const float* src = part + (int64_t)b * parts * width + c;
  double s = 0.0;
  if (has)
    for (int i = q; i < parts; i += W * AHEAD) {
      float x[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) x[k] = i + k * W < parts ? src[(i + k * W) * width] : 0.f;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) s += (double)x[k];
    }
  lds[q][lane] = s;
  __syncthreads();
  if (has && q == 0) {
#pragma unroll
    for (int k = 1; k < W; ++k) s += lds[k][lane];
    if (which < 4) out[(int64_t)b * E + (c - which * (int64_t)E)] = (float)s;
    else out[b] = (float)s;
  }
}

constexpr int GN_MAX_E = 16384;
int gn_rows(int E) { return E <= 64 ? 32 : E <= 256 ? 8 : E <= 512 ? 4 : 1; }     // rows of a workgroup
// workgroups of a model in the backward call: as many as are resident at once, `per` on each of the 256 compute units
int gn_blocks(int B, int R, int E, int per) {
  const int rows = (R + gn_rows(E) - 1) / gn_rows(E);
  int most = 256 * (E <= 512 ? per : E <= 1024 ? 2 * per : E <= 2048 ? per : 1);
  most /= B;
  if (most < 32) most = 32;
  if (most > GN_MAX_BLOCKS) most = GN_MAX_BLOCKS;
  return rows < most ? rows : most;
}

int gn_check(int B, int R, int E, int dtype, int norm) {
  if (B <= 0 || R <= 0 || E <= 0 || !valid_dtype(dtype) || (norm != HFTA_NORM_RMS && norm != HFTA_NORM_LAYER)) return HFTA_EINVAL;
  if (E > GN_MAX_E || B > 65535) return HFTA_EUNSUPPORTED;
  const int64_t threads = E <= 512 ? 256 : E <= 1024 ? 128 : E <= 2048 ? 256 : E <= 4096 ? 512 : 1024;       // of a workgroup
  const int64_t blocks = ((int64_t)R + gn_rows(E) - 1) / gn_rows(E);
  return blocks > 0xffffff || blocks * threads > 0xffffffff ? HFTA_EUNSUPPORTED : HFTA_OK;
}

// pieces of a thread and threads of a row; the other template arguments
#define GN_LAUNCH(kernel, EL, TPR, ...) \
  hipLaunchKernelGGL((kernel<T, EL / Piece16<T>::N, TPR, __VA_ARGS__>), grid, dim3(gn_threads(TPR)), 0, st, a)
#define GN_FORMS(kernel, ...)                                       \
  if (a.E <= 64) GN_LAUNCH(kernel, 8, 8, __VA_ARGS__);              \
  else if (a.E <= 256) GN_LAUNCH(kernel, 8, 32, __VA_ARGS__);       \
  else if (a.E <= 512) GN_LAUNCH(kernel, 8, 64, __VA_ARGS__);       \
  else if (a.E <= 1024) GN_LAUNCH(kernel, 8, 128, __VA_ARGS__);     \
  else if (a.E <= 2048) GN_LAUNCH(kernel, 8, 256, __VA_ARGS__);     \
  else if (a.E <= 4096) GN_LAUNCH(kernel, 8, 512, __VA_ARGS__);     \
  else if (a.E <= 8192) GN_LAUNCH(kernel, 8, 1024, __VA_ARGS__);    \
  else GN_LAUNCH(kernel, 16, 1024, __VA_ARGS__);                    \
  return launch_status();

template <typename T, bool RMS, bool BLOCK> int gn_fwd(const GnArgs& a, int B, hipStream_t st) {
  const dim3 grid((unsigned)((a.R + gn_rows(a.E) - 1) / gn_rows(a.E)), (unsigned)B);
  GN_FORMS(gn_fwd_kernel, RMS, BLOCK)
}
template <typename T, bool RMS, bool BLOCK> int gn_bwd(const GnArgs& a, int B, hipStream_t st) {
  const dim3 grid((unsigned)a.blocks, (unsigned)B);
  GN_FORMS(gn_bwd_kernel, RMS, BLOCK, false)
}
template <typename T, bool RMS, bool BLOCK> int gn_bwd_bias(const GnArgs& a, int B, hipStream_t st) {
  const dim3 grid((unsigned)a.blocks, (unsigned)B);
  GN_FORMS(gn_bwd_kernel, RMS, BLOCK, true)
}
#define GN_PICK(fn, a, B, st)                                                                                                \
  (dtype == HFTA_BF16 ? (norm == HFTA_NORM_RMS ? (F ? fn<bf16_raw, true, true>(a, B, st) : fn<bf16_raw, true, false>(a, B, st))    \
                                               : (F ? fn<bf16_raw, false, true>(a, B, st) : fn<bf16_raw, false, false>(a, B, st))) \
                      : (norm == HFTA_NORM_RMS ? (F ? fn<float, true, true>(a, B, st) : fn<float, true, false>(a, B, st))          \
                                               : (F ? fn<float, false, true>(a, B, st) : fn<float, false, false>(a, B, st))))

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" {

int hfta_gated_residual_norm_fwd(int B, int R, int E, int dtype, int norm, const void* X, const void* F, const void* G, const float* w1,
                                 const float* b1, const float* res, const float* w2, const float* b2, float eps, void* S, void* Y,
                                 float* mean1, float* inv1, float* mean2, float* inv2, void* stream) {
  const int rc = gn_check(B, R, E, dtype, norm);
  const bool means = norm == HFTA_NORM_LAYER;
  if (rc == HFTA_EINVAL || !X || !w2 || !Y || !inv2 || !(eps >= 0.f) || (means && !mean2)) return HFTA_EINVAL;
  if (F ? (!w1 || !S || !inv1 || (means && !mean1)) : (G || w1 || b1 || res || S)) return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  GnArgs a{};
  a.X = X; a.F = F; a.G = G; a.w1 = w1; a.b1 = b1; a.res = res; a.w2 = w2; a.b2 = b2; a.eps = eps; a.S = S; a.Y = Y;
  a.m1 = mean1; a.i1 = inv1; a.m2 = mean2; a.i2 = inv2; a.R = R; a.E = E;
  return GN_PICK(gn_fwd, a, B, as_stream(stream));
}

size_t hfta_gated_residual_norm_bwd_workspace_bytes(int B, int R, int E) {
  if (gn_check(B, R, E, HFTA_F32, HFTA_NORM_RMS) != HFTA_OK) return 0;
  return (size_t)B * gn_blocks(B, R, E, 3) * (4 * (size_t)E + 4) * sizeof(float);
}

int hfta_gated_residual_norm_bwd(int B, int R, int E, int dtype, int norm, const void* X, const void* F, const void* G, const float* w1,
                                 const float* b1, const float* res, const float* w2, const float* mean1, const float* inv1,
                                 const float* mean2, const float* inv2, const void* dS, const void* dY, void* dX, void* dF, void* dG,
                                 float* dw1, float* db1, float* dw2, float* db2, float* dres, void* workspace, size_t ws_bytes,
                                 void* stream) {
  const int rc = gn_check(B, R, E, dtype, norm);
  const bool means = norm == HFTA_NORM_LAYER;
  if (rc == HFTA_EINVAL || !X || !w2 || !inv2 || !dY || !dX || !dw2 || (means && !mean2)) return HFTA_EINVAL;
  if (F ? (!w1 || !inv1 || (means && !mean1) || !dF || !dw1 || (!G != !dG) || (!b1 != !db1) || (!res && dres))
        : (G || w1 || b1 || res || dF || dG || dw1 || db1 || dres))
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 4 || ws_bytes < hfta_gated_residual_norm_bwd_workspace_bytes(B, R, E))
    return HFTA_EWORKSPACE;
  GnArgs a{};
  a.X = X; a.F = F; a.G = G; a.w1 = w1; a.b1 = b1; a.res = res; a.w2 = w2; a.dS = dS; a.dY = dY; a.dX = dX; a.dF = dF; a.dG = dG;
  a.m1 = const_cast<float*>(mean1); a.i1 = const_cast<float*>(inv1); a.m2 = const_cast<float*>(mean2); a.i2 = const_cast<float*>(inv2);
  a.R = R; a.E = E; a.part = reinterpret_cast<float*>(workspace);
  const bool bias = db1 || db2;
  a.blocks = gn_blocks(B, R, E, bias || dtype == HFTA_F32 ? 2 : 3);
  hipStream_t st = as_stream(stream);
  const int r = bias ? GN_PICK(gn_bwd_bias, a, B, st) : GN_PICK(gn_bwd, a, B, st);
  if (r != HFTA_OK) return r;
  const dim3 grid((unsigned)((4 * (int64_t)E + 1 + 63) / 64), (unsigned)B);
  hipLaunchKernelGGL(gn_add_kernel, grid, dim3(GN_ADD), 0, st, a.part, a.blocks, E, dw2, db2, dw1, db1, dres);
  return launch_status();
}

}  // extern "C"
