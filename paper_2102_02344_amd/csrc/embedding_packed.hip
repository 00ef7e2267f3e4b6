// Embedding of packed sequences and the gradient of its table by sorted tokens (fusion rules table row "Embedding").
//
//   out_r = scale table[idx_r] + pos[r - start of r's sequence];   dtable_v = scale * sum of dY_r over the rows with idx_r = v
//
// Both are bound by memory.  The lookup reads and writes rows in 16-byte pieces.  The gradient sorts each model's rows by
// token -- stable, so that the rows of a token keep their order and the sum is the same bit for bit on every run --
// and walks the sorted rows in stretches of SORT_CH, a wavefront per stretch and 256 columns with eight rows in flight.  A
// token whose rows lie within one stretch is written from there; of a longer run each stretch leaves a partial sum, and
// the workgroup of the stretch in which it begins adds them, in order, so that a frequent token (padding, the first words
// of a text) costs no serial walk.  The sort: digits of at most eight bits from the lowest on, each a count per
// 4096 rows, a scan and a scatter.
#include "packed_rows.h"

namespace hfta {
namespace {

// ------------------------------------------------------------------ lookup
constexpr int EP_ROWS = 32;
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void ep_fwd_kernel(const T* __restrict__ table, const int32_t* __restrict__ idx,
                                                     const int32_t* __restrict__ off, int nseq, const float* __restrict__ pos,
                                                     T* __restrict__ out, int R, int V, int E, int S, float scale) {
  constexpr int EPP = VEC ? 16 / (int)sizeof(T) : 1;
  __shared__ PackedRows<EP_ROWS> pr;
  __shared__ int tok[EP_ROWS], place[EP_ROWS];
  const int b = blockIdx.y, t = threadIdx.x, t0 = blockIdx.x * EP_ROWS;
  pr.template scan<256>(off + (int64_t)b * (nseq + 1), nseq, R, t0);
  if (t < EP_ROWS) {
    int lo, hi;
    const bool in = pr.range(t0, t, lo, hi);
    tok[t] = in ? min(max(idx[(int64_t)b * R + t0 + t], 0), V - 1) : -1;
    place[t] = min(t0 + t - lo, S - 1);
  }
  __syncthreads();
  const int ppr = E / EPP, rows = min(EP_ROWS, R - t0), dr = 256 / ppr, dc = 256 - dr * ppr;
  int r = t / ppr, c = t - r * ppr;
  while (r < rows) {
    if (tok[r] >= 0) {
      const T* src = table + ((int64_t)b * V + tok[r]) * E + c * EPP;
      T* dst = out + ((int64_t)b * R + t0 + r) * E + c * EPP;
      const float* pp = pos ? pos + (int64_t)place[r] * E + c * EPP : nullptr;
      if constexpr (VEC) {
        union { uint4 u; T e[EPP]; } x;
        x.u = *reinterpret_cast<const uint4*>(src);
        float p[EPP];
#pragma unroll
        for (int q = 0; q < EPP / 4; ++q) {
          const float4 v = pp ? *reinterpret_cast<const float4*>(pp + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f);
          p[4 * q] = v.x; p[4 * q + 1] = v.y; p[4 * q + 2] = v.z; p[4 * q + 3] = v.w;
        }
#pragma unroll
        for (int e = 0; e < EPP; ++e) x.e[e] = Elem<T>::from_f32(fmaf(scale, Elem<T>::to_f32(x.e[e]), p[e]));
        *reinterpret_cast<uint4*>(dst) = x.u;
      } else {
        Elem<T>::store(dst, fmaf(scale, Elem<T>::load(src), pp ? *pp : 0.f));
      }
    }
    r += dr;
    c += dc;
    if (c >= ppr) { c -= ppr; ++r; }
  }
}

// ------------------------------------------------------------------ sort
constexpr int SORT_BLK = 4096, SORT_BINS = 256, SORT_CH = 32, SORT_SLICE = 256;

// Token of a row: its index, or V (past every token) for a row outside the sequences.  The first pass reads the indices,
// later ones the pairs (token, row) that the pass before left.
struct SortIn {
  const int32_t *idx, *off;
  const uint2* pairs;
  int nseq, R, V;
  __device__ __forceinline__ uint2 operator()(int b, int i) const {
    if (pairs) return pairs[(int64_t)b * R + i];
    const int v = min(max(idx[(int64_t)b * R + i], 0), V - 1);
    const bool in = !off || (i >= off[(int64_t)b * (nseq + 1)] && i < off[(int64_t)b * (nseq + 1) + nseq]);
    return make_uint2(in ? (uint32_t)v : (uint32_t)V, (uint32_t)i);
  }
};

// hist [B][bins][blocks]: how many of a block's rows have each digit
__global__ __launch_bounds__(256) void sort_count_kernel(SortIn in, uint32_t* __restrict__ hist, int shift, uint32_t mask) {
  __shared__ uint32_t h[SORT_BINS];
  const int b = blockIdx.y, t = threadIdx.x, blk = blockIdx.x, nblk = gridDim.x;
  h[t] = 0;
  __syncthreads();
  const int lo = blk * SORT_BLK, hi = min(in.R, lo + SORT_BLK);
  for (int i = lo + t; i < hi; i += 256) atomicAdd(&h[(in(b, i).x >> shift) & mask], 1u);
  __syncthreads();
  if (t <= (int)mask) hist[((int64_t)b * (mask + 1) + t) * nblk + blk] = h[t];
}

// exclusive sums over a model's n counts, in place: one workgroup of 1024 threads per model
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* __restrict__ hist, int n) {
  __shared__ uint32_t w[16];
  uint32_t* h = hist + (int64_t)blockIdx.x * n;
  const int t = threadIdx.x, lane = t & 63;
  uint32_t before = 0;
  for (int i0 = 0; i0 < n; i0 += 1024) {
    const int i = i0 + t;
    const uint32_t x = i < n ? h[i] : 0;
    uint32_t v = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(v, o, 64);
      if (lane >= o) v += y;
    }
    __syncthreads();
    if (lane == 63) w[t >> 6] = v;
    __syncthreads();
    uint32_t base = before;
    for (int k = 0; k < (t >> 6); ++k) base += w[k];
    if (i < n) h[i] = base + v - x;
    for (int k = 0; k < 16; ++k) before += w[k];
  }
}

// Each wavefront takes 1024 neighbouring rows of a block, 64 at a time: a row's place is its digit's first place in this
// block, plus the rows of that digit in the wavefronts before, plus those met so far, plus the lanes below.
__global__ __launch_bounds__(256) void sort_scatter_kernel(SortIn in, const uint32_t* __restrict__ hist, uint2* __restrict__ out,
                                                           int shift, int bits) {
  __shared__ uint32_t cnt[4][SORT_BINS];
  const int b = blockIdx.y, t = threadIdx.x, lane = t & 63, wave = t >> 6, blk = blockIdx.x, nblk = gridDim.x;
  const uint32_t mask = (1u << bits) - 1u;
#pragma unroll
  for (int k = 0; k < 4; ++k) cnt[k][t] = 0;
  __syncthreads();
  const int lo = blk * SORT_BLK + wave * (SORT_BLK / 4), hi = min(in.R, lo + SORT_BLK / 4);
  for (int i = lo + lane; i < hi; i += 64) atomicAdd(&cnt[wave][(in(b, i).x >> shift) & mask], 1u);
  __syncthreads();
  if (t <= (int)mask) {
    uint32_t at = hist[((int64_t)b * (mask + 1) + t) * nblk + blk];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = cnt[k][t];
      cnt[k][t] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int i0 = lo; i0 < hi; i0 += 64) {           // (the same number of steps for all lanes)
    const int i = i0 + lane;
    const bool ok = i < hi;
    const uint2 p = ok ? in(b, i) : make_uint2(0, 0);
    const uint32_t dg = (p.x >> shift) & mask;
    unsigned long long same = __ballot(ok);
    for (int k = 0; k < bits; ++k) {
      const unsigned long long m = __ballot((dg >> k) & 1u);
      same &= (dg >> k) & 1u ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    const uint32_t at = cnt[wave][dg];
    __builtin_amdgcn_wave_barrier();
    if (ok) {
      out[(int64_t)b * in.R + at + rank] = p;
      if (rank == 0) cnt[wave][dg] = at + (uint32_t)__popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ------------------------------------------------------------------ sums of the sorted rows
__global__ __launch_bounds__(256) void ep_zero_kernel(float* __restrict__ p, int64_t n) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
    if (i + 4 <= n) *reinterpret_cast<float4*>(p + i) = make_float4(0.f, 0.f, 0.f, 0.f);
    else for (int64_t k = i; k < n; ++k) p[k] = 0.f;
  }
}

// four columns of a row
template <typename T, bool VEC> struct EpCols {
  union { T e[4]; uint2 h; uint4 w; };
  __device__ __forceinline__ void load(const T* row, int c, int E) {
    if constexpr (VEC) {
      if constexpr (sizeof(T) == 2) h = *reinterpret_cast<const uint2*>(row + c);
      else w = *reinterpret_cast<const uint4*>(row + c);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = row[min(c + k, E - 1)];
    }
  }
};
template <bool VEC> __device__ __forceinline__ void ep_store(float* dst, int c, int E, const float (&x)[4], float f) {
  if constexpr (VEC) {
    *reinterpret_cast<float4*>(dst + c) = make_float4(f * x[0], f * x[1], f * x[2], f * x[3]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < E) dst[c + k] = f * x[k];
  }
}

// part [B][chunks][2][E]: of a stretch, the sum of the run that came in from the stretch before (0), and of the run that
// begins here and goes on behind it (1)
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void ep_sum_kernel(const T* __restrict__ dY, const uint2* __restrict__ sorted, float* __restrict__ dtable,
                                                     float* __restrict__ part, int R, int V, int E, int chunks, float scale) {
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const int ch = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = blockIdx.z * SORT_SLICE + 4 * lane;
  if (ch >= chunks) return;
  const int lo = ch * SORT_CH, n = min(SORT_CH, R - lo);
  const uint2* s = sorted + (int64_t)b * R;
  // lane i: the stretch's i-th pair; the token before and behind it
  const uint2 p = s[min(lo + lane, R - 1)];
  const uint32_t prev = lo ? s[lo - 1].x : 0xffffffffu, next = lo + n < R ? s[lo + n].x : 0xffffffffu;
  const T* dy = dY + (int64_t)b * R * E;
  float* pa = part + ((int64_t)b * chunks + ch) * 2 * E;
  const bool mine = c < E;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  uint32_t cur = __builtin_amdgcn_readfirstlane(p.x);
  bool from_before = cur == prev;
  auto flush = [&](bool goes_on) {
    if (!mine || cur >= (uint32_t)V) return;
    if (from_before) ep_store<VEC>(pa, c, E, acc, 1.f);
    else if (goes_on) ep_store<VEC>(pa + E, c, E, acc, 1.f);
    else ep_store<VEC>(dtable + ((int64_t)b * V + cur) * E, c, E, acc, scale);
  };
  for (int i0 = 0; i0 < n; i0 += 8) {
    EpCols<T, VEC> x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint32_t r = __builtin_amdgcn_readlane(p.y, min(i0 + u, n - 1));
      if (mine) x[u].load(dy + (int64_t)r * E, c, E);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i0 + u >= n) continue;
      const uint32_t k = __builtin_amdgcn_readlane(p.x, i0 + u);
      if (k != cur) {
        flush(false);
        cur = k;
        from_before = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += Elem<T>::to_f32(x[u].e[e]);
    }
  }
  flush(cur == next);
}

// The workgroup of the stretch in which a run begins adds what the stretches left of it: a wavefront per quarter of them.
template <bool VEC>
__global__ __launch_bounds__(256) void ep_join_kernel(const uint2* __restrict__ sorted, const float* __restrict__ part,
                                                      float* __restrict__ dtable, int R, int V, int E, int chunks, float scale) {
  __shared__ float sh[4][SORT_SLICE];
  const int b = blockIdx.y, ch = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.z * SORT_SLICE + 4 * lane;
  const uint2* s = sorted + (int64_t)b * R;
  const int lo = ch * SORT_CH, hi = lo + SORT_CH;
  if (hi >= R) return;
  const uint32_t v = s[hi - 1].x;
  if (v >= (uint32_t)V || s[hi].x != v || (s[lo].x == v && lo && s[lo - 1].x == v)) return;      // nothing goes on, or it began before
  int a = hi, z = R;                                  // the run's end: the first position behind it
  while (a < z) {
    const int mid = a + ((z - a) >> 1);
    if (s[mid].x == v) a = mid + 1;
    else z = mid;
  }
  const int last = (a - 1) / SORT_CH, m = last - ch;  // stretches ch + 1 .. last hold the rest
  const int per = (m + 3) / 4, from = ch + 1 + wave * per, to = min(last + 1, from + per);
  const bool mine = c < E;
  const float* pb = part + (int64_t)b * chunks * 2 * E;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  if (mine) {
    if (wave == 0) {
      EpCols<float, VEC> x;
      x.load(pb + ((int64_t)ch * 2 + 1) * E, c, E);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = x.e[e];
    }
    for (int k0 = from; k0 < to; k0 += 8) {
      EpCols<float, VEC> x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u].load(pb + (int64_t)min(k0 + u, to - 1) * 2 * E, c, E);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (k0 + u < to) {
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += x[u].e[e];
        }
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sh[wave][4 * lane + e] = acc[e];
  __syncthreads();
  if (wave == 0 && mine) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = (sh[0][4 * lane + e] + sh[1][4 * lane + e]) + (sh[2][4 * lane + e] + sh[3][4 * lane + e]);
    ep_store<VEC>(dtable + ((int64_t)b * V + v) * E, c, E, acc, scale);
  }
}

int ep_check(int B, int R, int V, int E, int dtype) {
  if (B <= 0 || R <= 0 || V <= 0 || E <= 0 || !valid_dtype(dtype)) return HFTA_EINVAL;
  return B > 65535 || E > 65535 * SORT_SLICE || R > 0x7fffffff - SORT_BLK ? HFTA_EUNSUPPORTED : HFTA_OK;
}

struct SortPlan {
  int nblk, chunks, passes, bits;
  size_t pairs, hist, part, total;                    // bytes: one buffer of pairs, the counts, the partial sums
  SortPlan(int B, int R, int V, int E) {
    nblk = R / SORT_BLK + (R % SORT_BLK != 0);
    chunks = R / SORT_CH + (R % SORT_CH != 0);
    int b = 1;
    while ((V >> b) > 0) ++b;                         // tokens 0 .. V
    passes = (b + 7) / 8;
    bits = (b + passes - 1) / passes;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    pairs = up((size_t)B * R * sizeof(uint2));
    hist = up((size_t)B * ((size_t)1 << bits) * nblk * 4);
    part = up((size_t)B * chunks * 2 * E * 4);
    total = 2 * pairs + hist + part;
  }
};

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" {

int hfta_embedding_packed_fwd(int B, int R, int V, int E, int nseq, int dtype, const void* table, const int32_t* idx,
                              const int32_t* seq_offsets, float scale, const float* pos, int S, void* out, void* stream) {
  const int rc = ep_check(B, R, V, E, dtype);
  if (rc == HFTA_EINVAL || nseq <= 0 || !table || !idx || !seq_offsets || !out || (pos && S <= 0)) return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  const int epp = dtype == HFTA_BF16 ? 8 : 4;
  const bool vec = E % epp == 0 && ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const dim3 grid((unsigned)((R + EP_ROWS - 1) / EP_ROWS), (unsigned)B);
  hipStream_t st = as_stream(stream);
  if (!pos) S = 1;
#define EP_FWD(T, VEC) hipLaunchKernelGGL((ep_fwd_kernel<T, VEC>), grid, dim3(256), 0, st, (const T*)table, idx, seq_offsets, nseq, pos, \
                                          (T*)out, R, V, E, S, scale)
  if (dtype == HFTA_BF16) { if (vec) EP_FWD(bf16_raw, true); else EP_FWD(bf16_raw, false); }
  else { if (vec) EP_FWD(float, true); else EP_FWD(float, false); }
#undef EP_FWD
  return launch_status();
}

size_t hfta_embedding_bwd_sorted_workspace_bytes(int B, int R, int V, int E) {
  return ep_check(B, R, V, E, HFTA_F32) == HFTA_OK ? SortPlan(B, R, V, E).total : 0;
}

int hfta_embedding_bwd_sorted(int B, int R, int V, int E, int nseq, int dtype, const void* dY, const int32_t* idx,
                              const int32_t* seq_offsets, float scale, float* dtable, void* workspace, size_t ws_bytes,
                              void* stream) {
  const int rc = ep_check(B, R, V, E, dtype);
  if (rc == HFTA_EINVAL || (seq_offsets && nseq <= 0) || !dY || !idx || !dtable) return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  const SortPlan pl(B, R, V, E);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 || ws_bytes < pl.total) return HFTA_EWORKSPACE;
  unsigned char* w = (unsigned char*)workspace;
  uint2* pairs[2] = {(uint2*)w, (uint2*)(w + pl.pairs)};
  uint32_t* hist = (uint32_t*)(w + 2 * pl.pairs);
  float* part = (float*)(w + 2 * pl.pairs + pl.hist);
  hipStream_t st = as_stream(stream);
  const int64_t n = (int64_t)B * V * E;
  hipLaunchKernelGGL(ep_zero_kernel, dim3((unsigned)(n / 1024 > 65535 ? 65535 : n / 1024 + 1)), dim3(256), 0, st, dtable, n);
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  SortIn in{idx, seq_offsets, nullptr, nseq, R, V};
  const dim3 grid((unsigned)pl.nblk, (unsigned)B);
  for (int k = 0; k < pl.passes; ++k) {
    const int shift = k * pl.bits;
    hipLaunchKernelGGL(sort_count_kernel, grid, dim3(256), 0, st, in, hist, shift, (1u << pl.bits) - 1u);
    if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
    hipLaunchKernelGGL(sort_scan_kernel, dim3((unsigned)B), dim3(1024), 0, st, hist, (1 << pl.bits) * pl.nblk);
    if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
    hipLaunchKernelGGL(sort_scatter_kernel, grid, dim3(256), 0, st, in, hist, pairs[k & 1], shift, pl.bits);
    if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
    in.pairs = pairs[k & 1];
  }
  const int es = dtype == HFTA_BF16 ? 2 : 4;
  const bool vec = E % 4 == 0 && reinterpret_cast<uintptr_t>(dY) % (4 * es) == 0 && reinterpret_cast<uintptr_t>(dtable) % 16 == 0;
  const dim3 gs((unsigned)((pl.chunks + 3) / 4), (unsigned)B, (unsigned)((E + SORT_SLICE - 1) / SORT_SLICE));
  const dim3 gj((unsigned)pl.chunks, (unsigned)B, gs.z);
#define EP_SUM(T, VEC) hipLaunchKernelGGL((ep_sum_kernel<T, VEC>), gs, dim3(256), 0, st, (const T*)dY, in.pairs, dtable, part, R, V, E, \
                                          pl.chunks, scale)
  if (dtype == HFTA_BF16) { if (vec) EP_SUM(bf16_raw, true); else EP_SUM(bf16_raw, false); }
  else { if (vec) EP_SUM(float, true); else EP_SUM(float, false); }
#undef EP_SUM
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  if (vec) hipLaunchKernelGGL(ep_join_kernel<true>, gj, dim3(256), 0, st, in.pairs, part, dtable, R, V, E, pl.chunks, scale);
  else hipLaunchKernelGGL(ep_join_kernel<false>, gj, dim3(256), 0, st, in.pairs, part, dtable, R, V, E, pl.chunks, scale);
  return launch_status();
}

}  // extern "C"
