// Embedding of packed sequences and the gradient of its table by sorted tokens (fusion rules table row "Embedding").
//
//   out_r = scale table[idx_r] + pos[r - start of r's sequence];   dtable_v = scale * sum of dY_r over the rows with idx_r = v
//
// Both are bound by memory.  The lookup reads and writes rows in 16-byte pieces.  The gradient sorts each model's rows by
// token -- stable, so that the rows of a token keep their order and the sum is the same bit for bit on every run --
// and walks the sorted rows in stretches of SORT_CH, a wavefront per stretch and 256 columns with sixteen rows in flight.  A
// token whose rows end in the stretch behind their first at the latest is written from there; of a longer run each stretch
// leaves a partial sum, and a workgroup adds them, in order, so that a frequent token (padding, the first words
// of a text) costs no serial walk.  The sort: digits of at most eight bits from the lowest on, a count and a scatter each.
//
// Measured, 2 x 60000 bf16 rows of 1024 columns, 32001 tokens: lookup 105 us (4.7 TB/s), sort 31 in four launches, sums 112, long runs 14; 8
// x 8192 rows of 256, 8192 tokens: 13, 18, 18 and 6, launches and chains of loads.
#include "packed_rows.h"

namespace hfta {
namespace {

// ------------------------------------------------------------------ lookup
constexpr int EP_ROWS = 32;
template <typename T, bool VEC, bool POS>
__global__ __launch_bounds__(256) void ep_fwd_kernel(const T* __restrict__ table, const int32_t* __restrict__ idx,
                                                     const int32_t* __restrict__ off, int nseq, const float* __restrict__ pos,
                                                     T* __restrict__ out, int R, int V, int E, int S, float scale) {
  constexpr int EPP = VEC ? 16 / (int)sizeof(T) : 1, EP_FLY = VEC ? 2 : 8;      // pieces of a thread in flight
  __shared__ PackedRows<EP_ROWS> pr;
  __shared__ int tok[EP_ROWS], place[EP_ROWS];
  const int b = blockIdx.y, t = threadIdx.x, t0 = blockIdx.x * EP_ROWS;
  pr.template scan<256>(off + (int64_t)b * (nseq + 1), nseq, R, t0);
  if (t < EP_ROWS) {
    int lo, hi;
    const bool in = pr.range(t0, t, lo, hi);
    tok[t] = in ? min(max(idx[(int64_t)b * R + t0 + t], 0), V - 1) : -1;
    place[t] = in ? min(t0 + t - lo, S - 1) : 0;
  }
  __syncthreads();
  const int ppr = E / EPP, rows = min(EP_ROWS, R - t0), dr = 256 / ppr, dc = 256 - dr * ppr;
  int r = t / ppr, c = t - r * ppr;
  union Piece { uint4 u; T e[VEC ? EPP : 16 / (int)sizeof(T)]; };
  while (r < rows) {
    Piece x[EP_FLY];
    float p[EP_FLY][EPP];
    int at[EP_FLY], col[EP_FLY];
#pragma unroll
    for (int j = 0; j < EP_FLY; ++j) {
      const int rj = min(r, rows - 1), v = tok[rj];
      at[j] = r < rows && v >= 0 ? r : -1;
      col[j] = c * EPP;
      const T* src = table + ((int64_t)b * V + max(v, 0)) * E + col[j];      // (loads without a branch: all in flight)
      const float* pp = pos + (int64_t)place[rj] * E + col[j];
      if constexpr (VEC) {
        x[j].u = *reinterpret_cast<const uint4*>(src);
#pragma unroll
        for (int q = 0; q < EPP / 4; ++q) {
          const float4 v = POS ? *reinterpret_cast<const float4*>(pp + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f);
          p[j][4 * q] = v.x; p[j][4 * q + 1] = v.y; p[j][4 * q + 2] = v.z; p[j][4 * q + 3] = v.w;
        }
      } else {
        x[j].e[0] = *src;
        p[j][0] = POS ? *pp : 0.f;
      }
      r += dr;
      c += dc;
      if (c >= ppr) { c -= ppr; ++r; }
    }
#pragma unroll
    for (int j = 0; j < EP_FLY; ++j) {
      if (at[j] < 0) continue;
#pragma unroll
      for (int e = 0; e < EPP; ++e) x[j].e[e] = Elem<T>::from_f32(fmaf(scale, Elem<T>::to_f32(x[j].e[e]), p[j][e]));
      T* dst = out + ((int64_t)b * R + t0 + at[j]) * E + col[j];
      if constexpr (VEC) *reinterpret_cast<uint4*>(dst) = x[j].u;
      else *dst = x[j].e[0];
    }
  }
}

// ------------------------------------------------------------------ sort
// Blocks add up the counts of those before them by themselves up to SORT_SELF of them, else a launch does (one workgroup per model).  The whole gradient
// of 8 columns and 8192 tokens, us by blocks and by a launch: 8 models of 20000 rows 41 / 47, 65536 76 / 79, 131072 157 / 130, 500000 1000 / 440; one model of 65536
// rows 34 / 43, 131072 46 / 63, 500000 145 / 182.
constexpr int SORT_BLK = 1024, SORT_BINS = 256, SORT_SELF = 64, SORT_ONE = 2048, SORT_CH = 32, SORT_SLICE = 256;

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

// lanes whose digit is this lane's, of those with `ok`
__device__ __forceinline__ unsigned long long sort_same(uint32_t dg, bool ok, int bits) {
  unsigned long long same = __ballot(ok);
  for (int k = 0; k < bits; ++k) {
    const unsigned long long m = __ballot((dg >> k) & 1u);
    same &= (dg >> k) & 1u ? m : ~m;
  }
  return same;
}
// exclusive sum over 256 threads; w: four words of LDS.  Two barriers.
__device__ __forceinline__ uint32_t sort_scan256(uint32_t x, uint32_t* w) {
  const int t = threadIdx.x, lane = t & 63;
  uint32_t v = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  if (lane == 63) w[t >> 6] = v;
  __syncthreads();
  uint32_t base = 0;
  for (int k = 0; k < (t >> 6); ++k) base += w[k];
  __syncthreads();
  return base + v - x;
}

// hist [B][bins][blocks]: how many of a block's rows have each digit.  (Counted by the scatter before, with atomics in memory, the
// frequent tokens made that launch 62 us where both are 21: 2 x 60000 rows.)
__global__ __launch_bounds__(256) void sort_count_kernel(SortIn in, uint32_t* __restrict__ hist, int shift, uint32_t mask) {
  __shared__ uint32_t h[SORT_BINS];
  const int b = blockIdx.y, blk = blockIdx.x, nblk = gridDim.x, t = threadIdx.x;
  h[t] = 0;
  __syncthreads();
  const int lo = blk * SORT_BLK, hi = min(in.R, lo + SORT_BLK);
#pragma unroll
  for (int k = 0; k < SORT_BLK / 256; ++k)
    if (lo + k * 256 + t < hi) atomicAdd(&h[(in(b, lo + k * 256 + t).x >> shift) & mask], 1u);
  __syncthreads();
  if (t <= (int)mask) hist[((int64_t)b * (mask + 1) + t) * nblk + blk] = h[t];
}

// exclusive sums over a model's n counts, in place: one workgroup of 1024 threads per model, eight counts each
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* __restrict__ hist, int n) {
  __shared__ uint32_t w[16];
  uint32_t* h = hist + (int64_t)blockIdx.x * n;
  const int t = threadIdx.x, lane = t & 63;
  uint32_t before = 0;
  for (int i0 = 0; i0 < n; i0 += 8192) {
    uint32_t x[8], sum = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = i0 + t * 8 + k;
      x[k] = i < n ? h[i] : 0;
      sum += x[k];
    }
    uint32_t v = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(v, o, 64);
      if (lane >= o) v += y;
    }
    __syncthreads();
    if (lane == 63) w[t >> 6] = v;
    __syncthreads();
    uint32_t at = before + v - sum;
    for (int k = 0; k < 16; ++k) {
      if (k < (t >> 6)) at += w[k];
      before += w[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = i0 + t * 8 + k;
      if (i < n) h[i] = at;
      at += x[k];
    }
  }
}

// Each wavefront takes a quarter of a block's rows, 64 at a time: a row's place is its digit's first place in this
// block, plus the rows of that digit in the wavefronts before, plus those met so far, plus the lanes below.  SELF: hist holds counts,
// and the block adds up those of lower digits and of earlier blocks itself (few blocks).
template <bool SELF>
__global__ __launch_bounds__(256) void sort_scatter_kernel(SortIn in, const uint32_t* __restrict__ hist, uint2* __restrict__ out,
                                                           int shift, int bits) {
  constexpr int PER = SORT_BLK / 4;
  __shared__ uint32_t cnt[4][SORT_BINS], w[4];
  const int b = blockIdx.y, blk = blockIdx.x, nblk = gridDim.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t mask = (1u << bits) - 1u;
  const int lo = blk * SORT_BLK + wave * PER;
  const uint32_t* hd = hist + ((int64_t)b * (mask + 1) + min(t, (int)mask)) * nblk;
  uint2 p[PER / 64];
#pragma unroll
  for (int k = 0; k < PER / 64; ++k) p[k] = lo + k * 64 + lane < in.R ? in(b, lo + k * 64 + lane) : make_uint2(0, 0);
#pragma unroll
  for (int k = 0; k < 4; ++k) cnt[k][t] = 0;
  uint32_t at = 0;
  if (SELF) {
    uint32_t all = 0;
    for (int k0 = 0; k0 < nblk; k0 += 8) {
      uint32_t c[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) c[k] = k0 + k < nblk ? hd[k0 + k] : 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        all += c[k];
        at += k0 + k < blk ? c[k] : 0;
      }
    }
    at += sort_scan256(t <= (int)mask ? all : 0, w);   // (its barriers stand between the clearing of cnt and the counts)
  } else {
    at = hd[blk];
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < PER / 64; ++k)
    if (lo + k * 64 + lane < in.R) atomicAdd(&cnt[wave][(p[k].x >> shift) & mask], 1u);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t c = cnt[k][t];
    cnt[k][t] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER / 64; ++k) {
    const bool ok = lo + k * 64 + lane < in.R;
    const uint32_t dg = (p[k].x >> shift) & mask;
    const unsigned long long same = sort_same(dg, ok, bits);
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    const uint32_t base = cnt[wave][dg];
    __builtin_amdgcn_wave_barrier();
    if (ok) {
      out[(int64_t)b * in.R + base + rank] = p[k];
      if (rank == 0) cnt[wave][dg] = base + (uint32_t)__popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Up to SORT_ONE rows: all passes in one workgroup's LDS.  (With 8192 rows, eight steps of 64 a wavefront: no sooner than the
// launches above, 27 us on 8 x 8192 rows.)
__global__ __launch_bounds__(1024) void sort_one_kernel(SortIn in, uint2* __restrict__ out, int passes, int bits) {
  constexpr int PER = SORT_ONE / 16;
  __shared__ uint2 buf[SORT_ONE];
  __shared__ uint32_t cnt[16][SORT_BINS], w[4];
  const int b = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6, lo = wave * PER;
  const uint32_t mask = (1u << bits) - 1u;
  uint2 p[PER / 64];
#pragma unroll
  for (int k = 0; k < PER / 64; ++k) p[k] = lo + k * 64 + lane < in.R ? in(b, lo + k * 64 + lane) : make_uint2(0, 0);
  for (int q = 0; q < passes; ++q) {
    const int shift = q * bits;
#pragma unroll
    for (int k = 0; k < 4; ++k) (&cnt[0][0])[k * 1024 + t] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER / 64; ++k)
      if (lo + k * 64 + lane < in.R) atomicAdd(&cnt[wave][(p[k].x >> shift) & mask], 1u);
    __syncthreads();
    uint32_t all = 0;
    if (t < 256)
      for (int k = 0; k < 16; ++k) all += cnt[k][t];
    uint32_t v = all;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(v, o, 64);
      if (lane >= o) v += y;
    }
    if (t < 256 && lane == 63) w[wave] = v;
    __syncthreads();
    if (t < 256) {
      uint32_t at = v - all;
      for (int k = 0; k < wave; ++k) at += w[k];
      for (int k = 0; k < 16; ++k) {
        const uint32_t c = cnt[k][t];
        cnt[k][t] = at;
        at += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER / 64; ++k) {
      const bool ok = lo + k * 64 + lane < in.R;
      const uint32_t dg = (p[k].x >> shift) & mask;
      const unsigned long long same = sort_same(dg, ok, bits);
      const int rank = __popcll(same & ((1ull << lane) - 1ull));
      const uint32_t base = cnt[wave][dg];
      __builtin_amdgcn_wave_barrier();
      if (ok) {
        buf[base + rank] = p[k];
        if (rank == 0) cnt[wave][dg] = base + (uint32_t)__popcll(same);
      }
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER / 64; ++k)
      if (lo + k * 64 + lane < in.R) p[k] = buf[lo + k * 64 + lane];
  }
#pragma unroll
  for (int k = 0; k < PER / 64; ++k)
    if (lo + k * 64 + lane < in.R) out[(int64_t)b * in.R + lo + k * 64 + lane] = p[k];
}

// ------------------------------------------------------------------ sums of the sorted rows
// four columns of a row from c on: in pieces c .. c + 3, else c, c + 64, .., so that a wavefront's lanes read next to each other
// (sums of 5 x 2888 rows of 665 bf16 columns: 23 us, with four side by side 34)
template <bool VEC> __device__ __forceinline__ int ep_col(int slice, int lane) { return slice * SORT_SLICE + (VEC ? 4 * lane : lane); }
template <typename T, bool VEC> struct EpCols {
  union { T e[4]; uint2 h; uint4 w; };
  __device__ __forceinline__ void load(const T* row, int c, int E) {
    if constexpr (VEC) {
      if constexpr (sizeof(T) == 2) h = *reinterpret_cast<const uint2*>(row + c);
      else w = *reinterpret_cast<const uint4*>(row + c);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = row[min(c + 64 * k, E - 1)];
    }
  }
};
template <bool VEC> __device__ __forceinline__ void ep_store(float* dst, int c, int E, const float (&x)[4], float f) {
  if constexpr (VEC) {
    *reinterpret_cast<float4*>(dst + c) = make_float4(f * x[0], f * x[1], f * x[2], f * x[3]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + 64 * k < E) dst[c + 64 * k] = f * x[k];
  }
}

// A run that begins in a stretch and ends in it or the next one is added by the wavefront of the first.  part [B][chunks][2][E]: of a
// stretch, the sum of a longer run's rows that came in from the stretch before (0), and that begin here (1).  `beside`: wavefronts of
// a workgroup on one stretch, next to each other in its columns, so that a wide row is read at once.  Workgroups behind the `sums` that
// add clear the rows of tokens that no row has: a workgroup takes 64 tokens, a lane
// looks for one each, and each wavefront clears a quarter of those missing (64 tokens a wavefront: 371 fp32 rows of 681 columns, 411 tokens, 22 us
// instead of 10; 2 x 60000 of 1024, 32001 tokens, 123 instead of 112).  (Clearing the whole table beside the sort writes the
// other rows twice: 278 us with the lookup for 2 x 60000 rows, 32001 tokens of 1024 columns.)
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void ep_sum_kernel(const T* __restrict__ dY, const uint2* __restrict__ sorted, float* __restrict__ dtable,
                                                     float* __restrict__ part, int R, int V, int E, int chunks, int beside, int sums, float scale) {
  constexpr int FLY = 16;                             // rows in flight
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= sums) {
    const uint2* s = sorted + (int64_t)b * R;
    const int64_t step = (int64_t)(gridDim.x - sums) * gridDim.z * 64;
    for (int64_t v0 = ((int64_t)(blockIdx.x - sums) * gridDim.z + blockIdx.z) * 64; v0 < V; v0 += step) {
      const int64_t v = v0 + lane;
      int a = 0, z = R;                               // the first place whose token is not below v
      while (a < z) {
        const int mid = a + ((z - a) >> 1);
        if ((int64_t)s[mid].x < v) a = mid + 1;
        else z = mid;
      }
      unsigned long long none = __ballot(v < V && (lane & 3) == wave && (a == R || (int64_t)s[a].x != v));
      const float zero[4] = {};
      for (; none; none &= none - 1) {
        float* row = dtable + ((int64_t)b * V + v0 + __builtin_ctzll(none)) * E;
        for (int c = ep_col<VEC>(0, lane); c < E; c += SORT_SLICE) ep_store<VEC>(row, c, E, zero, 1.f);
      }
    }
    return;
  }
  const int ch = blockIdx.x * (4 / beside) + wave / beside, c = ep_col<VEC>(blockIdx.z * beside + wave % beside, lane);
  if (ch >= chunks) return;
  const int lo = ch * SORT_CH, n = min(SORT_CH, R - lo);
  const uint2* s = sorted + (int64_t)b * R;
  auto at = [&](int i) { return i >= 0 && i < R ? s[i] : make_uint2(0xffffffffu, 0); };
  // the stretch before and this one, and the 64 rows behind it, a lane each; one row more in front
  const uint2 pa = at(lo - SORT_CH + lane), pb = at(lo + SORT_CH + lane);
  const uint32_t far = at(lo - SORT_CH - 1).x;
  auto key = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane(i < 32 ? pa.x : pb.x, i < 32 ? 32 + i : i - 32); };
  const uint32_t k0 = key(0), kn = (uint32_t)__builtin_amdgcn_readlane(pa.x, 31 + n);
  const unsigned long long head = __ballot(pa.x == k0), tail = __ballot(pb.x == kn);     // bits 32..63 of head: this stretch
  if (k0 >= (uint32_t)V) return;                      // rows of no sequence: the last of the order
  const bool from_before = (head >> 31) & 1;
  const bool whole = (uint32_t)(head >> 32) == 0xffffffffu && key(32) == k0;             // and goes on
  const bool head_long = from_before && (whole || ((uint32_t)head == 0xffffffffu && far == k0));
  int i = from_before && !head_long ? __builtin_ctzll(~(head >> 32) | 0x100000000ull) : 0;
  const bool goes_on = n == SORT_CH && (tail & 1) && !(from_before && k0 == kn);
  const bool tail_long = goes_on && ((tail >> 32) & 1);
  const int end = goes_on && !tail_long ? SORT_CH + __builtin_ctzll(~tail) : n;
  const T* dy = dY + (int64_t)b * R * E;
  float* pt = part + ((int64_t)b * chunks + ch) * 2 * E;
  const bool mine = c < E;
  float acc[4] = {};
  uint32_t cur = i < end ? key(i) : 0xffffffffu;
  bool first = head_long;                             // the current run is the one from before
  auto flush = [&](bool last) {
    if (!mine || cur >= (uint32_t)V) return;
    if (first) ep_store<VEC>(pt, c, E, acc, 1.f);
    else if (last && tail_long) ep_store<VEC>(pt + E, c, E, acc, 1.f);
    else ep_store<VEC>(dtable + ((int64_t)b * V + cur) * E, c, E, acc, scale);
  };
  for (; i < end; i += FLY) {
    EpCols<T, VEC> x[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const int j = min(i + u, end - 1);
      const uint32_t r = (uint32_t)__builtin_amdgcn_readlane(j < 32 ? pa.y : pb.y, j < 32 ? 32 + j : j - 32);
      if (mine) x[u].load(dy + (int64_t)r * E, c, E);
    }
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      if (i + u >= end) continue;
      const uint32_t k = key(i + u);
      if (k != cur) {
        flush(false);
        cur = k;
        first = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += Elem<T>::to_f32(x[u].e[e]);
    }
  }
  if (cur != 0xffffffffu) flush(true);
}

// The longer runs: a workgroup looks at four stretches, and of a run that begins in one of them adds what the stretches left, a
// wavefront per quarter of them.
template <bool VEC>
__global__ __launch_bounds__(256) void ep_join_kernel(const uint2* __restrict__ sorted, const float* __restrict__ part,
                                                      float* __restrict__ dtable, int R, int V, int E, int chunks, float scale) {
  constexpr int FLY = 8;
  __shared__ float sh[4][SORT_SLICE];
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = ep_col<VEC>(blockIdx.z, lane);
  const uint2* s = sorted + (int64_t)b * R;
  const bool mine = c < E;
  const float* pt = part + (int64_t)b * chunks * 2 * E;
  auto at = [&](int i) { return i >= 0 && i < R ? s[i].x : 0xffffffffu; };
  for (int k = 0; k < 4; ++k) {                       // (the same for the whole workgroup)
    const int ch = blockIdx.x * 4 + k, lo = ch * SORT_CH, hi = lo + SORT_CH;
    if (hi + SORT_CH >= R) break;
    const uint32_t v = at(hi - 1);
    const bool here = v < (uint32_t)V && at(hi) == v && at(hi + SORT_CH) == v && !(at(lo) == v && at(lo - 1) == v);
    if (!here) continue;
    int m = 0;                                        // stretches behind this one that begin inside the run
    for (;; m += 64) {
      const int x = ch + 1 + m + lane;
      const unsigned long long in = __ballot(x < chunks && s[min(x, chunks - 1) * SORT_CH].x == v);
      if (in != ~0ull) { m += __builtin_ctzll(~in); break; }
    }
    const int per = (m + 3) / 4, from = ch + 1 + wave * per, to = min(ch + 1 + m, from + per);
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
      if (wave == 0) {
        EpCols<float, VEC> x;
        x.load(pt + ((int64_t)ch * 2 + 1) * E, c, E);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = x.e[e];
      }
      for (int j = from; j < to; j += FLY) {
        EpCols<float, VEC> x[FLY];
#pragma unroll
        for (int u = 0; u < FLY; ++u) x[u].load(pt + (int64_t)min(j + u, to - 1) * 2 * E, c, E);
#pragma unroll
        for (int u = 0; u < FLY; ++u)
          if (j + u < to) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += x[u].e[e];
          }
      }
    }
    __syncthreads();                                  // the last run's sums have been read
#pragma unroll
    for (int e = 0; e < 4; ++e) sh[wave][4 * lane + e] = acc[e];
    __syncthreads();
    if (wave == 0 && mine) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = (sh[0][4 * lane + e] + sh[1][4 * lane + e]) + (sh[2][4 * lane + e] + sh[3][4 * lane + e]);
      ep_store<VEC>(dtable + ((int64_t)b * V + v) * E, c, E, acc, scale);
    }
  }
}

int ep_check(int B, int R, int V, int E, int dtype) {
  if (B <= 0 || R <= 0 || V <= 0 || E <= 0 || !valid_dtype(dtype)) return HFTA_EINVAL;
  return B > 65535 || E > 65535 * SORT_SLICE || R > 1 << 28 || V > 1 << 30 ? HFTA_EUNSUPPORTED : HFTA_OK;     // (a launch has fewer than 2^32 threads)
}

struct SortPlan {
  int nblk, chunks, passes, bits;
  bool one, self;
  size_t pairs, hist, part, total;                    // bytes: one buffer of pairs, the counts, the partial sums
  SortPlan(int B, int R, int V, int E) {
    nblk = R / SORT_BLK + (R % SORT_BLK != 0);
    chunks = R / SORT_CH + (R % SORT_CH != 0);
    int b = 1;
    while ((V >> b) > 0) ++b;                         // tokens 0 .. V
    passes = (b + 7) / 8;
    bits = (b + passes - 1) / passes;
    one = R <= SORT_ONE;
    self = nblk <= SORT_SELF;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    pairs = up((size_t)B * R * sizeof(uint2));
    hist = one ? 0 : up((size_t)B * ((size_t)1 << bits) * nblk * 4);
    part = up((size_t)B * chunks * 2 * E * 4);
    total = (one ? 1 : 2) * pairs + hist + part;
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
  if (rc != HFTA_OK || nseq > PACKED_MAX) return HFTA_EUNSUPPORTED;
  const int epp = dtype == HFTA_BF16 ? 8 : 4;
  const bool vec = E % epp == 0 && ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const dim3 grid((unsigned)((R + EP_ROWS - 1) / EP_ROWS), (unsigned)B);
  hipStream_t st = as_stream(stream);
  if (!pos) S = 1;
#define EP_FWD(T, VEC, POS) hipLaunchKernelGGL((ep_fwd_kernel<T, VEC, POS>), grid, dim3(256), 0, st, (const T*)table, idx, seq_offsets, nseq, pos, \
                                               (T*)out, R, V, E, S, scale)
#define EP_FWD_AS(T)                                                                                \
  do {                                                                                              \
    if (vec) { if (pos) EP_FWD(T, true, true); else EP_FWD(T, true, false); }                       \
    else { if (pos) EP_FWD(T, false, true); else EP_FWD(T, false, false); }                         \
  } while (0)
  if (dtype == HFTA_BF16) EP_FWD_AS(bf16_raw);
  else EP_FWD_AS(float);
#undef EP_FWD_AS
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
  if (rc != HFTA_OK || (seq_offsets && nseq > PACKED_MAX)) return HFTA_EUNSUPPORTED;
  const SortPlan pl(B, R, V, E);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 || ws_bytes < pl.total) return HFTA_EWORKSPACE;
  unsigned char* w = (unsigned char*)workspace;
  uint2* pairs[2] = {(uint2*)w, (uint2*)(w + (pl.one ? 0 : pl.pairs))};
  w += (pl.one ? 1 : 2) * pl.pairs;
  uint32_t* hist = (uint32_t*)w;
  float* part = (float*)(w + pl.hist);
  hipStream_t st = as_stream(stream);
  SortIn in{idx, seq_offsets, nullptr, nseq, R, V};
  if (pl.one) {
    hipLaunchKernelGGL(sort_one_kernel, dim3((unsigned)B), dim3(1024), 0, st, in, pairs[0], pl.passes, pl.bits);
    if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
    in.pairs = pairs[0];
  } else {
    const dim3 grid((unsigned)pl.nblk, (unsigned)B);
    for (int k = 0; k < pl.passes; ++k) {
      hipLaunchKernelGGL(sort_count_kernel, grid, dim3(256), 0, st, in, hist, k * pl.bits, (1u << pl.bits) - 1u);
      if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
      if (!pl.self) {
        hipLaunchKernelGGL(sort_scan_kernel, dim3((unsigned)B), dim3(1024), 0, st, hist, (1 << pl.bits) * pl.nblk);
        if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
      }
      if (pl.self) hipLaunchKernelGGL(sort_scatter_kernel<true>, grid, dim3(256), 0, st, in, hist, pairs[k & 1], k * pl.bits, pl.bits);
      else hipLaunchKernelGGL(sort_scatter_kernel<false>, grid, dim3(256), 0, st, in, hist, pairs[k & 1], k * pl.bits, pl.bits);
      if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
      in.pairs = pairs[k & 1];
    }
  }
  const int es = dtype == HFTA_BF16 ? 2 : 4;
  const bool vec = E % 4 == 0 && reinterpret_cast<uintptr_t>(dY) % (4 * es) == 0 && reinterpret_cast<uintptr_t>(dtable) % 16 == 0;
  const int slices = (E + SORT_SLICE - 1) / SORT_SLICE, beside = slices > 2 ? 4 : slices;
  const int sums = (pl.chunks + 4 / beside - 1) / (4 / beside), groups = (slices + beside - 1) / beside;
  // (sums are at most 2^23 and a launch has fewer than 2^24 workgroups in x: of more than 2^28 tokens a workgroup clears several times 64)
  const int64_t clears = (V + (int64_t)64 * groups - 1) / (64 * groups);
  const dim3 gs((unsigned)(sums + (clears < 1 << 22 ? clears : 1 << 22)), (unsigned)B, (unsigned)groups);
  const dim3 gj((unsigned)((pl.chunks + 3) / 4), (unsigned)B, (unsigned)slices);
#define EP_SUM(T, VEC) hipLaunchKernelGGL((ep_sum_kernel<T, VEC>), gs, dim3(256), 0, st, (const T*)dY, in.pairs, dtable, part, R, V, E, \
                                          pl.chunks, beside, sums, scale)
  if (dtype == HFTA_BF16) { if (vec) EP_SUM(bf16_raw, true); else EP_SUM(bf16_raw, false); }
  else { if (vec) EP_SUM(float, true); else EP_SUM(float, false); }
#undef EP_SUM
  if (launch_status() != HFTA_OK) return HFTA_ELAUNCH;
  if (pl.chunks <= 2) return HFTA_OK;                 // no run is longer than two stretches
  if (vec) hipLaunchKernelGGL(ep_join_kernel<true>, gj, dim3(256), 0, st, in.pairs, part, dtable, R, V, E, pl.chunks, scale);
  else hipLaunchKernelGGL(ep_join_kernel<false>, gj, dim3(256), 0, st, in.pairs, part, dtable, R, V, E, pl.chunks, scale);
  return launch_status();
}

}  // extern "C"
