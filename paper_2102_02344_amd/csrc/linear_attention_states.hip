// Linear attention: the states that blocks of tiles hand on, and their sums along the sequences (linear_attention.h).
#include "linear_attention.h"

namespace hfta {
namespace {

// What the sequence of a block's last row, if it goes on, has gathered in this block
template <typename T, int D, bool VEC, bool PIECES> __global__ __launch_bounds__(4 * D, (sizeof(T) == 2 || D < 128 ? 4 : 2)) void la_block_kernel(LaArgs a) {
  typedef LaStage<T, D, VEC> Stage;
  constexpr int NT = LaWave<D>::NT;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[2 * Stage::BYTES];
  __shared__ PackedRows<LA_T> pr;
  __shared__ __attribute__((aligned(16))) float pw[LA_T], wt[LA_T];
  const LaWave<D> wv;
  const LaPlace at(a, true);
  const LaJob& J = a.job[at.job];
  const int rev = J.rev, t = threadIdx.x, hk = at.h;
  const int first = at.blk * a.per, last = first + a.per - 1;
  if (at.blk == a.blocks - 1) return;                            // hands on nothing
  const int32_t* off = a.off + (int64_t)at.b * (a.nseq + 1);
  const float ld = la_decay(a.ld[(int64_t)at.b * a.Hkv + hk]);
  if (t < LA_T) pw[t] = la_pow(ld, t);
  const int a0 = (rev ? a.tiles - 1 - last : last) * LA_T, j = rev ? 0 : LA_T - 1;
  pr.template scan<NT>(off, a.nseq, a.R, a0);
  int start, end;
  const bool on = a0 + j < a.R && pr.range(a0, j, start, end) && (rev ? start < a0 : end > a0 + LA_T);
  const int begin = rev ? a.tiles * LA_T - end : start;          // of the sequence, in the order of the walk
  if (t == 0 && hk == 0) a.spans[((int64_t)at.job * a.B + at.b) * a.blocks + at.blk] = !on ? 0 : begin < first * LA_T ? 2 : 1;
  if (!on) return;
  la_f4 s[D / 16];
#pragma unroll
  for (int n = 0; n < D / 16; ++n) s[n] = la_f4{0.f, 0.f, 0.f, 0.f};
  const bool fresh = begin >= first * LA_T;
  if (PIECES && fresh && J.S0) la_load_state<T, D>(s, J, a, at.b, la_sequence(off, a.nseq, a0 + j), hk, wv);
  const T* pb = pk_at<T>(J.B, J.bs, at.b, hk * J.gb);
  const T* pc = pk_at<T>(J.C, J.cs, at.b, hk * J.gb);
  Stage sb, sc;
  sb.init(J.bs.r, a.d, rev);
  sc.init(J.cs.r, a.d, rev);
  const la_lds lb = (la_lds)tiles, lc = (la_lds)tiles + Stage::BYTES;
  const float f64 = la_faded(ld, LA_T);
#pragma unroll 1
  for (int tile = fresh ? begin / LA_T : first; tile <= last; ++tile) {
    const int c0 = max(begin - tile * LA_T, 0), m0 = (rev ? a.tiles - 1 - tile : tile) * LA_T;
    // against the order, what comes in behind the last row has not faded when that row is taken
    const int n = LA_T - c0 - (PIECES && J.S0 && rev && fresh && tile == begin / LA_T ? 1 : 0);
    la_fade(s, n == LA_T ? f64 : la_faded(ld, n));
#pragma unroll 1
    for (int h = 0; h < J.gb; ++h) {
      __syncthreads();
      if (t < LA_T) wt[t] = t >= c0 ? pw[LA_T - 1 - t] : 0.f;
      sb.fetch(lb, pb + h * J.bs.h + m0 * J.bs.r, J.bs.r, a.R - m0, a.d, rev);
      sc.fetch(lc, pc + h * J.cs.h + m0 * J.cs.r, J.cs.r, a.R - m0, a.d, rev);
      la_land<VEC>();
      if (c0 > 0) {                                              // (what stands in rows of other sequences does not matter)
        la_clear<T, D>(lb, c0);
        __syncthreads();
      }
      la_update<T, D, false, PIECES>(s, lb, lc, wt, 0, LA_T, wv);
    }
  }
  float* sums = a.sums + ((((int64_t)at.job * a.B + at.b) * a.Hkv + hk) * a.blocks + at.blk) * (D * D);
#pragma unroll
  for (int kt = 0; kt < D / 16; ++kt) *la_sum<D>(sums, wv.cs, kt, wv.lane) = s[kt];
}

// Sums along the sequences, in place: a thread has four entries of a state and walks the blocks, eight blocks' loads in flight
__global__ __launch_bounds__(256) void la_scan_kernel(LaArgs a, int entries) {
  constexpr int AHEAD = 8;
  const int64_t state = blockIdx.y;                              // job, model, key head
  const int64_t jb = state / a.Hkv;
  const int hk = (int)(state % a.Hkv), b = (int)(jb % a.B);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= entries) return;
  const float f = la_faded(la_decay(a.ld[(int64_t)b * a.Hkv + hk]), a.per * LA_T);
  const bool less = f > 0.f;
  const int* spans = a.spans + jb * a.blocks;
  float4* p = reinterpret_cast<float4*>(a.sums) + (state * a.blocks) * entries + i;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < a.blocks - 1; k0 += AHEAD) {
    float4 v[AHEAD];
    int sp[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      sp[k] = k0 + k < a.blocks - 1 ? spans[k0 + k] : 0;
      if (sp[k]) v[k] = p[(int64_t)(k0 + k) * entries];
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (sp[k]) {
        if (sp[k] == 2) {
          v[k].x += fmaf(s.x, f, less ? 0.f : s.x);
          v[k].y += fmaf(s.y, f, less ? 0.f : s.y);
          v[k].z += fmaf(s.z, f, less ? 0.f : s.z);
          v[k].w += fmaf(s.w, f, less ? 0.f : s.w);
          p[(int64_t)(k0 + k) * entries] = v[k];
        }
        s = v[k];
      }
  }
}

template <typename T, int D> int launch(const LaArgs& a, const LaForm& f, hipStream_t st) {
  const dim3 grid((unsigned)LaPlace::count(a, true)), block(LaWave<D>::NT);
  if (f.vec && f.pieces) hipLaunchKernelGGL((la_block_kernel<T, D, true, true>), grid, block, 0, st, a);
  else if (f.vec) hipLaunchKernelGGL((la_block_kernel<T, D, true, false>), grid, block, 0, st, a);
  else if (f.pieces) hipLaunchKernelGGL((la_block_kernel<T, D, false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((la_block_kernel<T, D, false, false>), grid, block, 0, st, a);
  if (a.mode == LA_SCANNED) {
    const int entries = D * D / 4;
    hipLaunchKernelGGL(la_scan_kernel, dim3((entries + 255) / 256, (unsigned)(a.nsums * a.B * a.Hkv)), dim3(256), 0, st, a, entries);
  }
  return launch_status();
}

}  // namespace

int la_states(const LaArgs& a, const LaForm& f, hipStream_t st) { return PK_BY_SIZE(launch); }

}  // namespace hfta
