// Linear attention with decays over packed sequences: the entry points (linear_attention.h).
#include "linear_attention.h"

namespace hfta {
namespace {

// Blocks of tiles: about LA_WANT of all heads together, which is two or three workgroups on each compute unit; half as many where a compute unit holds one
// (128 columns of fp32, which take 143 KB of LDS, or of bf16 with states, whose registers leave room for one) and in the backward call, whose three jobs run
// side by side (8 x 2048 rows, 4 heads of 64 bf16, both directions: 57 us with 512 for each job, 51 with 256, 62 with 170; 2 x 16384 rows, 8 heads of 128: 437,
// 412, 429).  With R their number only grows, so that the workspace for the most rows serves fewer.
constexpr int LA_MOST = 0x1fffff;        // query heads and blocks: a launch has fewer than 2^32 threads, three jobs of up to 512 for each
constexpr int LA_WANT = 512, LA_SCAN = 32 * 128 * 128, LA_FEW = 64 * 64, LA_SHORT = 512;
int la_check(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  if (B <= 0 || R <= 0 || nseq <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv || !valid_dtype(dtype) || R > 0x7fffffff - 4096) return HFTA_EINVAL;
  return d > 128 || nseq > PACKED_MAX || B > 65535 || (int64_t)B * Hq > LA_MOST ? HFTA_EUNSUPPORTED : HFTA_OK;
}
// Against the order a state is held divided by the scale, which is why that has to lie well inside the range of fp32
bool la_scale(float scale) { return scale >= 0x1p-32f && scale <= 0x1p32f; }
int64_t la_limit(int B, int Hq, int Hkv, int want) {
  const int64_t blocks = (int64_t)B * Hkv < want ? want / ((int64_t)B * Hkv) : 1, most = LA_MOST / ((int64_t)B * Hq);
  return blocks < most ? blocks : most;
}
void la_cut(LaArgs& a, int Hq, int dtype) {
  a.by_heads = PkDiv((uint32_t)(a.B * Hq));
  a.by_hq = PkDiv((uint32_t)Hq);
  a.by_key_heads = PkDiv((uint32_t)(a.B * a.Hkv));
  a.by_hkv = PkDiv((uint32_t)a.Hkv);
  bool states = false;
  for (int j = 0; j < a.jobs; ++j) states = states || a.job[j].S0 || a.job[j].S1;
  const int64_t most = la_limit(a.B, Hq, a.Hkv, a.jobs > 1 || (a.d > 64 && (dtype == HFTA_F32 || states)) ? LA_WANT / 2 : LA_WANT);
  a.tiles = (a.R + LA_T - 1) / LA_T;
  a.per = (int)((a.tiles + most - 1) / most);
  a.blocks = (a.tiles + a.per - 1) / a.per;
  // Short sequences are walked up to a block once more instead of summed, which saves the launches for states: 8 x 2048 rows, 4 heads of 64 bf16, both
  // directions: sequences of 200 rows 66 us with sums and 52 walked, of 400 63 and 59, of 800 75 and 80.  Backward each query head of a group is walked:
  // 3 x 930 rows, 12 heads of 80 over 3, backward alone walked or not: of 50 rows 62 and 66, of 100 69 and 68, of 200 85 and 76.  fp32 takes longer for a
  // tile, the more the wider (3 x 777, 3 heads of 48: of 100 rows 41 and 38, of 200 46 and 57).  One long sequence among short ones costs its tiles again in
  // each of its blocks, so that this is left to few rows (three quarters of the rows in one: 66 and 80, of 8192 rows 105 and 200).  Places of sequences that are empty count as
  // short ones: 8 models of 4 heads of 32, 300 places and all rows in one of them, forward: 2048 rows bf16 25 us with sums and 37 walked, 8192 rows 60 and 128, fp32 94
  // and 240; in 80 sequences of 100 instead 52 and 45, fp32 82 and 75.
  // Sums are added up by each block for itself while those before it are up to 2 MB (16384 rows of one sequence, both directions: 2 x 4 heads of 64, 64 blocks
  // forward: 136 us, with a launch that adds them along the sequences 158; 2 x 8 heads of 128, 32 blocks: 395 and 410; 2 x 4, 64 blocks: 296 and 249; 1 x 1,
  // 256 blocks: 1040 and 279).
  const int D = la_pad(a.d), rows = dtype == HFTA_F32 ? LA_SHORT / (D > 64 ? 8 : 4) : LA_SHORT;
  const int64_t again = (int64_t)(a.R / a.nseq) * (a.jobs > 1 ? Hq / a.Hkv : 1);
  a.mode = a.blocks == 1 ? LA_ALONE : (int64_t)a.tiles * D <= LA_FEW && again <= rows ? LA_WALK : a.blocks * D * D > LA_SCAN ? LA_SCANNED : LA_SUMS;
}
size_t la_workspace(int B, int R, int Hq, int Hkv, int d, int sums) {
  const int64_t tiles = (R + LA_T - 1) / LA_T, most = la_limit(B, Hq, Hkv, LA_WANT), n = tiles < most ? tiles : most;
  if (n == 1) return 0;
  const int64_t D = la_pad(d);
  return (size_t)(sums * n * B * Hkv * D * D * 4 + (sums * n * B * 4 + 15) / 16 * 16);
}
void la_place(LaArgs& a, void* workspace) {
  if (a.blocks == 1) return;
  const int64_t D = la_pad(a.d);
  a.sums = reinterpret_cast<float*>(workspace);
  a.spans = reinterpret_cast<int*>(a.sums + (int64_t)a.nsums * a.blocks * a.B * a.Hkv * D * D);
}
bool la_ws_ok(void* workspace, size_t have, size_t need) { return need == 0 || (workspace && reinterpret_cast<uintptr_t>(workspace) % 16 == 0 && have >= need); }
PkStr la_str(const int64_t* s) { return PkStr{s[0], s[1], s[2]}; }
// rows in whole 16-byte pieces: pointers, strides and head widths
bool la_vec(const LaArgs& a, int dtype, const void* const* p, int n) {
  const int64_t m = dtype == HFTA_BF16 ? 8 : 4;
  uintptr_t bits = 0;
  for (int i = 0; i < n; ++i) bits |= reinterpret_cast<uintptr_t>(p[i]);
  bool vec = a.d % m == 0 && bits % 16 == 0;
  for (int j = 0; j < a.jobs; ++j) {
    const PkStr* s[] = {&a.job[j].as, &a.job[j].bs, &a.job[j].cs, &a.job[j].os};
    for (const PkStr* x : s) vec = vec && x->b % m == 0 && x->r % m == 0 && x->h % m == 0 && x->r >= 0 && x->r <= PK_LD_MAX;
  }
  return vec;
}
int la_run(const LaArgs& a, int dtype, bool vec, hipStream_t st) {
  LaForm f{dtype == HFTA_BF16, vec, false};
  for (int j = 0; j < a.jobs; ++j) f.pieces = f.pieces || a.job[j].S0 || a.job[j].S1;
  if (a.mode == LA_SUMS || a.mode == LA_SCANNED) {
    const int rc = la_states(a, f, st);
    if (rc != HFTA_OK) return rc;
  }
  return la_main(a, f, st);
}

}  // namespace
}  // namespace hfta

using namespace hfta;

extern "C" {

size_t hfta_linear_attention_fwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  return la_check(B, R, nseq, Hq, Hkv, d, dtype) == HFTA_OK ? la_workspace(B, R, Hq, Hkv, d, 1) : 0;
}
size_t hfta_linear_attention_bwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  return la_check(B, R, nseq, Hq, Hkv, d, dtype) == HFTA_OK ? la_workspace(B, R, Hq, Hkv, d, 2) : 0;
}

int hfta_linear_attention_fwd(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3], const void* K,
                              const void* V, const int64_t kvs[3], const int32_t* seq_offsets, const float* log_decay, float scale,
                              const float* state_in, void* CTX, const int64_t cs[3], float* state_out, void* workspace, size_t ws_bytes,
                              void* stream) {
  const int rc = la_check(B, R, nseq, Hq, Hkv, d, dtype);
  if (rc == HFTA_EINVAL || !Q || !qs || !K || !V || !kvs || !seq_offsets || !log_decay || !(scale > 0.f) || !isfinite(1.f / scale) || !CTX || !cs ||
      (state_out && state_out == state_in))
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  if (!la_scale(scale)) return HFTA_EUNSUPPORTED;
  if (!la_ws_ok(workspace, ws_bytes, la_workspace(B, R, Hq, Hkv, d, 1))) return HFTA_EWORKSPACE;
  LaArgs a{};
  a.off = seq_offsets; a.ld = log_decay; a.B = B; a.R = R; a.nseq = nseq; a.Hkv = Hkv; a.d = d; a.jobs = a.nsums = 1;
  const PkStr q = la_str(qs), kv = la_str(kvs), c = la_str(cs);
  a.job[0] = LaJob{Q, K, V, CTX, q, kv, kv, c, state_in, state_out, 0, 0, Hq / Hkv, 1, scale, 1.f, 0, 0};
  la_cut(a, Hq, dtype);
  la_place(a, workspace);
  const void* p[] = {Q, K, V, CTX};
  return la_run(a, dtype, la_vec(a, dtype, p, 4), as_stream(stream));
}

int hfta_linear_attention_bwd(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, const void* Q, const int64_t qs[3], const void* K,
                              const void* V, const int64_t kvs[3], const int32_t* seq_offsets, const float* log_decay, float scale,
                              const float* state_in, const void* dCTX, const int64_t cs[3], const float* dstate_out, void* dQ,
                              const int64_t dqs[3], void* dK, void* dV, const int64_t dkvs[3], float* dstate_in, void* workspace,
                              size_t ws_bytes, void* stream) {
  const int rc = la_check(B, R, nseq, Hq, Hkv, d, dtype);
  if (rc == HFTA_EINVAL || !Q || !qs || !K || !V || !kvs || !seq_offsets || !log_decay || !(scale > 0.f) || !isfinite(1.f / scale) || !dCTX || !cs ||
      !dQ || !dqs || !dK || !dV || !dkvs || (dstate_in && dstate_in == dstate_out))
    return HFTA_EINVAL;
  if (rc != HFTA_OK) return rc;
  if (!la_scale(scale)) return HFTA_EUNSUPPORTED;
  if (!la_ws_ok(workspace, ws_bytes, la_workspace(B, R, Hq, Hkv, d, 2))) return HFTA_EWORKSPACE;
  LaArgs a{};
  a.off = seq_offsets; a.ld = log_decay; a.B = B; a.R = R; a.nseq = nseq; a.Hkv = Hkv; a.d = d; a.jobs = 3; a.nsums = 2;
  const PkStr q = la_str(qs), kv = la_str(kvs), c = la_str(cs), dq = la_str(dqs), dkv = la_str(dkvs);
  const int G = Hq / Hkv;
  a.job[0] = LaJob{dCTX, V, K, dQ, c, kv, kv, dq, state_in, nullptr, 0, 1, G, 1, scale, 1.f, 0, 0};
  a.job[1] = LaJob{K, Q, dCTX, dV, kv, q, c, dkv, dstate_out, dstate_in, 1, 0, 1, G, scale, scale, 1, 0};
  a.job[2] = LaJob{V, dCTX, Q, dK, kv, c, q, dkv, dstate_out, nullptr, 1, 1, 1, G, scale, scale, 1, 1};
  la_cut(a, Hq, dtype);
  la_place(a, workspace);
  const void* p[] = {Q, K, V, dCTX, dQ, dK, dV};
  return la_run(a, dtype, la_vec(a, dtype, p, 7), as_stream(stream));
}

}  // extern "C"
