// Rotary positions along one or several axes on packed rows (the positions of rows that the fusion rules table's row "Embedding" adds as
// a table, here as rotations of the query and key heads).
//
// A pair of columns (u, v) of a row is a complex number, multiplied by e^(i a) with a = pos[axis of the pair] freq[pair]; the backward
// call multiplies by e^(-i a).  Far positions make angles of many turns, of which fp32 keeps nothing behind the first few digits: the
// angle is formed in 64 bits, in turns, and only the rest of less than half a turn goes on in fp32.
//
// Bound by memory: a lane forms the angles of a piece of 16 bytes once and turns that piece in all heads of its row.  The first four heads are on
// their way while the angles are formed, and a head is fetched as one is stored: 2 x 40000 rows, 10 heads of 128 bf16, three axes: 90 to 96 us
// from card to card, 4.3 to 4.5 TB/s, against 114 with loads four heads at a time.  Where few rows would leave compute units without work the heads are
// split over workgroups too.
#include "packed_rows.h"
#include "pieces.h"

namespace hfta {
namespace {

struct RoStr { int64_t b, r, h; };
struct RoArgs {
  const void* X;
  void* Y;
  const int32_t *pos, *axis, *off;
  const float* freq;
  RoStr xs, ys;
  int R, nseq, H, d, naxes, pairs, inverse;
  int turned, items;               // pieces of a row that are turned, and with those that are only copied
  int lanes, rows, heads;          // lanes of a row, rows and heads of a workgroup
};

// a piece as it was loaded: 16 bytes, or N elements one by one
template <typename T, bool WIDE, int N> struct RoRaw {
  piece_u4 v;
  __device__ __forceinline__ void get(const T* p, int n) { v = Piece16<T>::raw(p, n); }
  __device__ __forceinline__ void values(float (&x)[N]) const { Piece16<T>::values(x, v); }
};
template <typename T, int N> struct RoRaw<T, false, N> {
  float v[N];
  __device__ __forceinline__ void get(const T* p, int n) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < n ? Elem<T>::load(p + e) : 0.f;
  }
  __device__ __forceinline__ void values(float (&x)[N]) const {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = v[e];
  }
};

template <typename T, bool WIDE, bool INTER>
__global__ __launch_bounds__(256) void ro_kernel(RoArgs a) {
  constexpr int N = WIDE ? Piece16<T>::N : INTER ? 2 : 1;        // columns of a piece
  constexpr int NP = INTER ? N / 2 : N;                          // pairs
  constexpr int AHEAD = 4;
  __shared__ PackedRows<256> pr;
  const int b = blockIdx.y, t0 = blockIdx.x * a.rows, rl = threadIdx.x / a.lanes, lane = threadIdx.x - rl * a.lanes, r = t0 + rl;
  bool in = rl < a.rows && r < a.R;
  int start = 0, end;
  if (a.off) {
    pr.template scan<256>(a.off + (int64_t)b * (a.nseq + 1), a.nseq, a.R, t0);
    if (in) in = pr.range(t0, rl, start, end);
  }
  if (!in) return;
  const int h0 = blockIdx.z * a.heads, h1 = min(h0 + a.heads, a.H);
  const T* x = reinterpret_cast<const T*>(a.X) + b * a.xs.b + r * a.xs.r;
  T* y = reinterpret_cast<T*>(a.Y) + b * a.ys.b + r * a.ys.r;
  const int32_t* pos = a.pos ? a.pos + ((int64_t)b * a.R + r) * a.naxes : nullptr;
  const float* freq = a.freq + (int64_t)b * a.pairs;
  auto put = [&](T* p, const float (&v)[N], int n) {
    if constexpr (WIDE) {
      Piece16<T>::store(p, v, n);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < n) Elem<T>::store(p + e, v[e]);
    }
  };
  for (int i = lane; i < a.items; i += a.lanes) {
    if (i >= a.turned) {                                         // columns behind the pairs
      const int c = 2 * a.pairs + (i - a.turned) * N, n = a.d - c;
      for (int h = h0; h < h1; ++h) {
        RoRaw<T, WIDE, N> raw;
        float v[N];
        raw.get(x + h * a.xs.h + c, n);
        raw.values(v);
        put(y + h * a.ys.h + c, v, n);
      }
      continue;
    }
    const int p0 = i * NP, n = min(NP, a.pairs - p0);            // pairs that are there
    const int cu = INTER ? 2 * p0 : p0, cv = a.pairs + p0, nu = INTER ? 2 * n : n;
    RoRaw<T, WIDE, N> ru[AHEAD], rv[AHEAD];
    auto load = [&](int k, int h) __attribute__((always_inline)) {
      const T* row = x + min(h, h1 - 1) * a.xs.h;                // (past the last head: once more, for nothing)
      ru[k].get(row + cu, nu);
      if constexpr (!INTER) rv[k].get(row + cv, n);
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) load(k, h0 + k);
    float co[NP], si[NP];
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int p = min(p0 + e, a.pairs - 1);
      const int ax = a.axis ? min(max(a.axis[p], 0), a.naxes - 1) : 0;
      const double turns = (double)(pos ? pos[ax] : r - start) * (double)freq[p] * 0.15915494309189533577;      // 1 / 2 pi
      float s, c;
      sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &c);
      co[e] = c;
      si[e] = a.inverse ? -s : s;
    }
    auto turn = [&](float (&u)[N], float (&v)[N]) {
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        float &s = INTER ? u[2 * e] : u[e], &t = INTER ? u[(2 * e + 1) % N] : v[e];
        const float su = s * co[e] - t * si[e], sv = t * co[e] + s * si[e];
        s = su;
        t = sv;
      }
    };
    for (int h = h0; h < h1; h += AHEAD) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        if (h + k >= h1) break;
        float u[N], v[N];
        ru[k].values(u);
        if constexpr (!INTER) rv[k].values(v);
        load(k, h + k + AHEAD);
        turn(u, v);
        T* row = y + (h + k) * a.ys.h;
        put(row + cu, u, nu);
        if constexpr (!INTER) put(row + cv, v, n);
      }
    }
  }
}

template <typename T> int ro_launch(RoArgs a, int B, bool wide, bool inter, hipStream_t st) {
  const int n = wide ? 16 / (int)sizeof(T) : inter ? 2 : 1, np = inter ? n / 2 : n;
  a.turned = (a.pairs + np - 1) / np;
  a.items = a.turned + (a.X == a.Y ? 0 : (a.d - 2 * a.pairs + n - 1) / n);
  a.lanes = a.items < 256 ? a.items : 256;
  a.rows = 256 / a.lanes;
  const int64_t blocks = ((int64_t)a.R + a.rows - 1) / a.rows;
  if (blocks > 0xffffff) return HFTA_EUNSUPPORTED;
  a.heads = a.H;
  while (a.heads > 1 && blocks * B * ((a.H + a.heads - 1) / a.heads) < 1024) a.heads = (a.heads + 1) / 2;
  const int64_t groups = (a.H + a.heads - 1) / a.heads;
  if (groups > 65535) return HFTA_EUNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)B, (unsigned)groups);
  if (wide && inter) hipLaunchKernelGGL((ro_kernel<T, true, true>), grid, dim3(256), 0, st, a);
  else if (wide) hipLaunchKernelGGL((ro_kernel<T, true, false>), grid, dim3(256), 0, st, a);
  else if (inter) hipLaunchKernelGGL((ro_kernel<T, false, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((ro_kernel<T, false, false>), grid, dim3(256), 0, st, a);
  return launch_status();
}

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" int hfta_rotary_packed(int B, int R, int nseq, int H, int d, int dtype, const void* X, const int64_t xs[3],
                                  const int32_t* positions, int naxes, const int32_t* axis, int pairs, const float* freq, int interleaved,
                                  const int32_t* seq_offsets, int inverse, void* Y, const int64_t ys[3], void* stream) {
  if (B <= 0 || R <= 0 || H <= 0 || d <= 0 || !valid_dtype(dtype) || !X || !xs || !Y || !ys || !freq || pairs <= 0 || pairs > d / 2 ||
      naxes <= 0 || (naxes > 1 && (!positions || !axis)) || (seq_offsets && nseq <= 0) || R > 0x7fffffff - 256)
    return HFTA_EINVAL;
  if (X == Y && (xs[0] != ys[0] || xs[1] != ys[1] || xs[2] != ys[2])) return HFTA_EINVAL;
  if (B > 65535 || (seq_offsets && nseq > PACKED_MAX)) return HFTA_EUNSUPPORTED;
  RoArgs a{};
  a.X = X; a.Y = Y; a.pos = positions; a.axis = axis; a.off = seq_offsets; a.freq = freq;
  a.xs = RoStr{xs[0], xs[1], xs[2]};
  a.ys = RoStr{ys[0], ys[1], ys[2]};
  a.R = R; a.nseq = nseq; a.H = H; a.d = d; a.naxes = naxes; a.pairs = pairs; a.inverse = inverse != 0;
  // A piece of pairs takes two loads of 16 bytes; with fewer pairs than half a piece holds an element at a time wastes less
  const bool wide = pairs * (interleaved ? 2 : 1) >= (dtype == HFTA_BF16 ? 8 : 4);
  if (dtype == HFTA_BF16) return ro_launch<bf16_raw>(a, B, wide, interleaved != 0, as_stream(stream));
  return ro_launch<float>(a, B, wide, interleaved != 0, as_stream(stream));
}
