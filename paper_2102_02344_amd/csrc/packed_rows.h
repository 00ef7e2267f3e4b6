// Packed sequences: a model's R rows hold sequences of any lengths back to back, seq_offsets [B][nseq + 1] their bounds.
//
// A workgroup that takes rows t0 .. t0 + ROWS - 1 finds each row's sequence without a search: every offset is read once,
// those inside the tile leave a bit per row, and what is needed of the others is the largest up to t0 and the smallest
// past the tile.  A row's sequence begins at the highest bit at or below it and ends at the next one.  Offsets are
// taken into [0, R]; in whatever order they come they are bounds, so no row is ever given to two sequences and nothing
// outside the tensors is addressed.  (Maxima, minima and bits: the order of the atomics does not matter.)  Where there are many
// offsets a wavefront finds the last one up to t0 first, sixty-four places a step, and those past the tile are not read either:
// attention of 65536 rows, 8 heads of 64, in 16384 sequences 152 -> 74 us, in 65536 418 -> 75.
#pragma once
#include "common.h"

namespace hfta {

constexpr int PACKED_MAX = (1 << 24) - 2;             // sequences of a model (a launch of a workgroup for each has fewer than 2^32 threads)

template <int ROWS> struct PackedRows {
  uint32_t mark[ROWS / 32];
  int lo, hi, first, last;

  // called by all NT threads; ends with a barrier
  template <int NT> __device__ __forceinline__ void scan(const int32_t* __restrict__ off, int nseq, int R, int t0) {
    const int t = threadIdx.x, end = t0 + ROWS - 1;
    const bool many = nseq > 4 * NT;
    int from = 0;
    if (many) {                                       // the last place at or below t0, or 0
      const int lane = t & 63;
      for (int n = nseq + 1; n > 64;) {
        const int step = (n + 63) >> 6;
        const int le = __popcll(__ballot(lane * step < n && off[min(from + lane * step, nseq)] <= t0));
        const int skip = max(le - 1, 0) * step;
        from += skip;
        n = min(step, n - skip);
      }
    }
    int next = from + t <= nseq ? off[from + t] : 0;
    for (int i = t; i < ROWS / 32; i += NT) mark[i] = 0;
    if (t == 0) { lo = -1; hi = 0x7fffffff; first = 0x7fffffff; last = -1; }
    __syncthreads();
    int vlo = -1, vhi = 0x7fffffff, vfirst = 0x7fffffff, vlast = -1;
    auto take = [&](int o) {
      o = min(max(o, 0), R);
      vfirst = min(vfirst, o);
      vlast = max(vlast, o);
      if (o <= t0) vlo = max(vlo, o);
      else if (o > end) vhi = min(vhi, o);
      else atomicOr(&mark[(o - t0) >> 5], 1u << ((o - t0) & 31));
    };
    if (many && t < 2) take(off[t ? nseq : 0]);
    for (int i = from + t; i <= nseq; i += NT) {
      const int o = next;
      if (i + NT <= nseq) next = off[i + NT];
      take(o);
      if (many && o > end) break;
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
      vlo = max(vlo, __shfl_xor(vlo, s, 64));
      vhi = min(vhi, __shfl_xor(vhi, s, 64));
      vfirst = min(vfirst, __shfl_xor(vfirst, s, 64));
      vlast = max(vlast, __shfl_xor(vlast, s, 64));
    }
    if ((t & 63) == 0) {
      atomicMax(&lo, vlo);
      atomicMin(&hi, vhi);
      atomicMin(&first, vfirst);
      atomicMax(&last, vlast);
    }
    __syncthreads();
  }

  // whether row t0 + i lies in a sequence, and that sequence's rows [start, end)
  __device__ __forceinline__ bool range(int t0, int i, int& start, int& end) const {
    start = end = 0;
    if (t0 + i < first || t0 + i >= last) return false;
    const int w0 = i >> 5;
    const uint32_t upto = (2u << (i & 31)) - 1u;
    start = lo;
    for (int w = w0; w >= 0; --w) {
      const uint32_t m = mark[w] & (w == w0 ? upto : 0xffffffffu);
      if (m) { start = t0 + 32 * w + 31 - __builtin_clz(m); break; }
    }
    end = hi;
    for (int w = w0; w < ROWS / 32; ++w) {
      const uint32_t m = mark[w] & (w == w0 ? ~upto : 0xffffffffu);
      if (m) { end = t0 + 32 * w + __builtin_ctz(m); break; }
    }
    return true;
  }
};

}  // namespace hfta
