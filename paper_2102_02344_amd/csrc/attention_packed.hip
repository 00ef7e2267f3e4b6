// Attention over packed sequences: the entry points (attention_packed.h).
#include "attention_packed.h"

namespace hfta {
namespace {

int pk_check(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, float scale) {
  if (B <= 0 || R <= 0 || nseq <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv || !valid_dtype(dtype) || !(scale > 0.f) ||
      isinf(scale * PK_LOG2E) || R > 0x7fffffff - 128)
    return HFTA_EINVAL;
  // (a launch has fewer than 2^32 threads; tiles are of at least 64 rows where there are many)
  return d > 128 || nseq > PACKED_MAX || (int64_t)B * Hq > 0xffffff / pk_tiles(R, 2 * PK_WT) ? HFTA_EUNSUPPORTED : HFTA_OK;
}
// Workgroups that share the sums of 64 keys, so that there are about 2048 of them: eight per compute unit, enough to even out the
// keys that many rows see with those that few do.  A part is at least eight tiles of 32 rows on average, since adding the parts is a launch
// that reads and writes them: 2 x 8192 rows, 3 sequences, 8 heads of 128 over 2: 886 us, with 4 parts 366 and 28 for adding them; 2 x 6442
// rows, 15 sequences, 6 heads of 64 over 3: 70, with 3 parts 45 and 11; 8 x 2048 rows, 12 sequences, 4 heads of 64: 26, with 2 parts 31 and
// 13; 4 x 3591 rows, 133 sequences, 8 heads of 128 over 2: 42, with 4 parts 50 and 22.  Where tiles of keys are fewer than compute units
// a part is two tiles, or one in fp32, whose products take four times as long: 3 x 777 rows, 5 sequences, 6 fp32 heads of 48 over
// 2: 141, with 8 parts 27 and 6; 3 x 201 rows, 8 sequences, 2 fp32 heads of 96 over 1: 48, with 5 parts 18 and 7; 2883 rows, 55 sequences, 4
// heads of 40 over 2: 25, with 4 parts 14 and 5.
constexpr int PK_WANT = 2048;
int pk_parts(int B, int R, int nseq, int Hq, int Hkv, int dtype) {
  const int64_t base = (int64_t)pk_tiles(R, 2 * PK_WT) * B * Hkv;
  const int64_t rows = R / nseq + 2 * PK_WT < R ? R / nseq + 2 * PK_WT : R, tiles = rows * (Hq / Hkv) / PK_WT;
  const int64_t least = base >= 256 ? 8 : dtype == HFTA_BF16 ? 2 : 1;
  int64_t p = PK_WANT / base;
  if (p > PK_PARTS_MAX) p = PK_PARTS_MAX;
  if (p > tiles / least) p = tiles / least;
  return p < 1 ? 1 : (int)p;
}
size_t pk_sums(int B, int R, int Hq) { return ((size_t)B * Hq * R * sizeof(float) + 255) / 256 * 256; }     // bytes of D
// Bytes of the backward's workspace: D, and the largest sums of parts that any call has with as many rows or fewer.  p parts need at most
// PK_WANT / p tiles, so there are p R words per column at most with R up to that; the rows and sequences of a batch change from step to step, and a
// workspace for the largest serves them all (two fp32 words for each of PK_WANT tiles' columns: 134 MB at d = 128).
size_t pk_workspace(int B, int R, int Hq, int Hkv, int d) {
  const int64_t heads = (int64_t)B * Hkv;
  size_t most = 0;
  for (int p = 2; p <= PK_PARTS_MAX; ++p) {
    const int64_t rows = 2 * PK_WT * (PK_WANT / p / heads);
    const size_t n = (size_t)p * (size_t)(rows < R ? rows : R);
    if (n > most) most = n;
  }
  return pk_sums(B, R, Hq) + most * 2 * (size_t)heads * d * sizeof(float);
}
void pk_places(PkArgs& a) {
  a.by_heads = PkDiv((uint32_t)(a.B * a.Hkv));
  a.by_hkv = PkDiv((uint32_t)a.Hkv);
  a.by_group = PkDiv((uint32_t)(a.Hq / a.Hkv));
  a.by_parts = PkDiv((uint32_t)a.parts);
}
constexpr int PK_SHORT = 128;      // rows of a sequence on average up to which D is made exact for dq too: more of D's error than of others
PkStr pk_str(const int64_t* s) { return s ? PkStr{s[0], s[1], s[2]} : PkStr{0, 0, 0}; }

// vec: rows in whole 16-byte pieces -- pointers, strides and head widths.
// split: where tiles of 128 rows are too few for the compute units, most of all where sequences are long and a tile has many keys.
// Then four times the workgroups each walk a quarter of the keys, at the price of loading keys for 32 rows at a time.  us as one tile and split,
// forward and backward: 3 x 777 rows, 5 sequences, 6 heads of 48 over 2 (126 tiles): bf16 10.5 / 7.6 and 33 / 30, fp32 25 / 16 and 63 / 53;
// 8 x 1452, 2 heads of 96 over 1 (192): bf16 33 / 26 and 102 / 105, fp32 192 / 122 and 475 / 351; 3 x 7290, 13 sequences, 2 heads
// of 40 (348): bf16 forward 28 / 21; 4096, 8 heads of 128 (256): bf16 85 / 66 and 259 /
// 260, fp32 538 / 363 and 1403 / 1101; the same in 30 sequences: bf16 15 / 19 and 42 / 65, fp32 48 / 72 and 135 / 168; 8 x 2048, 4 heads of 64 (512), 2
// sequences: bf16 29 / 31 and 95 / 104, fp32 135 / 103 and 384 / 327, in 12: fp32 44 / 50 and 127 / 140; 4 x 2048, 16 heads of 128 (1024): bf16
// 92 / 150 and 318 / 499, fp32 604 / 799 and 2023 / 2216.
bool pk_split(const PkArgs& a, int dtype, bool bwd) {
  const int64_t tiles = (int64_t)pk_tiles(a.R, 4 * PK_WT) * a.B * a.Hq;
  const bool longer = a.R / a.nseq >= 384;
  if (dtype == HFTA_BF16) return tiles < (longer && !bwd ? 400 : 192);
  return tiles < 256 || (longer && tiles * (a.d > 64 ? 2 : 1) < 1024);
}
PkForm pk_form(const PkArgs& a, int dtype, const void* const* p, int n, bool bwd) {
  const int64_t m = dtype == HFTA_BF16 ? 8 : 4;
  uintptr_t bits = 0;
  for (int i = 0; i < n; ++i) bits |= reinterpret_cast<uintptr_t>(p[i]);
  const PkStr* s[] = {&a.qs, &a.ks, &a.cs, &a.dqs, &a.dks};
  bool vec = a.d % m == 0 && bits % 16 == 0;
  for (const PkStr* x : s) vec = vec && x->b % m == 0 && x->r % m == 0 && x->h % m == 0 && x->r >= 0 && x->r <= PK_LD_MAX;
  return PkForm{dtype == HFTA_BF16, vec, vec && pk_split(a, dtype, bwd)};
}

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
  a.parts = 1;
  pk_places(a);
  const void* p[] = {Q, K, V, CTX};
  return pk_fwd(a, pk_form(a, dtype, p, 4, false), as_stream(stream));
}

size_t hfta_attention_packed_bwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  if (pk_check(B, R, nseq, Hq, Hkv, d, dtype, 1.f) != HFTA_OK) return 0;
  return pk_workspace(B, R, Hq, Hkv, d);
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
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 ||
      ws_bytes < hfta_attention_packed_bwd_workspace_bytes(B, R, nseq, Hq, Hkv, d, dtype))
    return HFTA_EWORKSPACE;
  PkArgs a{};
  a.Q = Q; a.K = K; a.V = V; a.dCTX = dCTX; a.off = seq_offsets; a.CTX = const_cast<void*>(CTX); a.LSE = const_cast<float*>(LSE);
  a.dQ = dQ; a.dK = dK; a.dV = dV; a.Dsum = reinterpret_cast<float*>(workspace);
  a.part = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(workspace) + pk_sums(B, R, Hq));
  a.parts = pk_parts(B, R, nseq, Hq, Hkv, dtype);
  a.twice = R / nseq <= PK_SHORT;
  a.qs = pk_str(qs); a.ks = pk_str(kvs); a.cs = pk_str(cs); a.dqs = pk_str(dqs); a.dks = pk_str(dkvs);
  a.B = B; a.R = R; a.nseq = nseq; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.causal = causal != 0; a.scale = scale;
  pk_places(a);
  const void* p[] = {Q, K, V, CTX, dCTX, dQ, dK, dV};
  hipStream_t st = as_stream(stream);
  const PkForm f = pk_form(a, dtype, p, 8, true);
  const int rq = pk_dq(a, f, st);
  return rq != HFTA_OK ? rq : pk_dkv(a, f, st);
}

}  // extern "C"
