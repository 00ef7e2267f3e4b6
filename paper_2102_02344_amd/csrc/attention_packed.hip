// Attention over packed sequences: the entry points (attention_packed.h).
#include "attention_packed.h"

namespace hfta {
namespace {

int pk_check(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype, float scale) {
  if (B <= 0 || R <= 0 || nseq <= 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || Hq % Hkv || !valid_dtype(dtype) || !(scale > 0.f) ||
      isinf(scale) || R > 0x7fffffff - 128)
    return HFTA_EINVAL;
  // (a launch has fewer than 2^32 threads; tiles are of at least 64 rows where there are many)
  return d > 128 || nseq > PACKED_MAX || (int64_t)B * Hq > 0xffffff / pk_tiles(R, 2 * PK_WT) ? HFTA_EUNSUPPORTED : HFTA_OK;
}
// Workgroups that share the sums of 64 keys, so that there are about 2048 of them: eight per compute unit, enough to even out the
// keys that many rows see with those that few do.  A part is at least 16 tiles of 32 rows on average, or two where the
// tiles of keys alone are fewer than two workgroups per compute unit.  2 x 8192 rows, 3 sequences, 8 heads of 128 over 2: 886 us, with
// 4 parts 381 and 25 for adding them; 3 x 777 rows, 5 sequences, 6 fp32 heads of 48 over 2: 141, with 7 parts 39 in all; 8 x 2048 rows, 12
// sequences, 4 heads of 64: 27 us, with 2 parts 31 and 13.
int pk_parts(int B, int R, int nseq, int Hq, int Hkv) {
  const int64_t base = (int64_t)pk_tiles(R, 2 * PK_WT) * B * Hkv, tiles = (int64_t)(R / nseq) * (Hq / Hkv) / 32;
  int64_t p = 2048 / base;
  if (p > PK_PARTS_MAX) p = PK_PARTS_MAX;
  if (p > tiles / (base < 512 ? 2 : 16)) p = tiles / (base < 512 ? 2 : 16);
  return p < 1 ? 1 : (int)p;
}
size_t pk_sums(int B, int R, int Hq) { return ((size_t)B * Hq * R * sizeof(float) + 255) / 256 * 256; }     // bytes of D
void pk_places(PkArgs& a) {
  a.by_heads = PkDiv((uint32_t)(a.B * a.Hkv));
  a.by_hkv = PkDiv((uint32_t)a.Hkv);
  a.by_group = PkDiv((uint32_t)(a.Hq / a.Hkv));
  a.by_parts = PkDiv((uint32_t)a.parts);
}
constexpr int PK_SHORT = 128;      // rows of a sequence on average up to which D is made exact for dq too: more of D's error than of others
PkStr pk_str(const int64_t* s) { return s ? PkStr{s[0], s[1], s[2]} : PkStr{0, 0, 0}; }

// vec: rows in whole 16-byte pieces -- pointers, strides and head widths.  split: tiles of 128 rows would be fewer than two
// workgroups per compute unit.  3 x 777 rows, 6 fp32 heads of 48 (126 tiles), forward and queries' backward: 40 and 55 us, 19 and 23 split;
// 8 x 2048 rows, 4 heads of 64 (512 tiles): 18 and 21, 24 and 36 split.
PkForm pk_form(const PkArgs& a, int dtype, const void* const* p, int n, int heads) {
  const int64_t m = dtype == HFTA_BF16 ? 8 : 4;
  uintptr_t bits = 0;
  for (int i = 0; i < n; ++i) bits |= reinterpret_cast<uintptr_t>(p[i]);
  const PkStr* s[] = {&a.qs, &a.ks, &a.cs, &a.dqs, &a.dks};
  bool vec = a.d % m == 0 && bits % 16 == 0;
  for (const PkStr* x : s) vec = vec && x->b % m == 0 && x->r % m == 0 && x->h % m == 0 && x->r >= 0 && x->r <= PK_LD_MAX;
  return PkForm{dtype == HFTA_BF16, vec, vec && (int64_t)pk_tiles(a.R, 4 * PK_WT) * a.B * heads < 512};
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
  return pk_fwd(a, pk_form(a, dtype, p, 4, Hq), as_stream(stream));
}

size_t hfta_attention_packed_bwd_workspace_bytes(int B, int R, int nseq, int Hq, int Hkv, int d, int dtype) {
  if (pk_check(B, R, nseq, Hq, Hkv, d, dtype, 1.f) != HFTA_OK) return 0;
  const int parts = pk_parts(B, R, nseq, Hq, Hkv);
  return pk_sums(B, R, Hq) + (parts > 1 ? (size_t)parts * 2 * B * R * Hkv * d * sizeof(float) : 0);
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
  a.parts = pk_parts(B, R, nseq, Hq, Hkv);
  a.twice = R / nseq <= PK_SHORT;
  a.qs = pk_str(qs); a.ks = pk_str(kvs); a.cs = pk_str(cs); a.dqs = pk_str(dqs); a.dks = pk_str(dkvs);
  a.B = B; a.R = R; a.nseq = nseq; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.causal = causal != 0; a.scale = scale;
  pk_places(a);
  const void* p[] = {Q, K, V, CTX, dCTX, dQ, dK, dV};
  hipStream_t st = as_stream(stream);
  const int rq = pk_dq(a, pk_form(a, dtype, p, 8, Hq), st);
  return rq != HFTA_OK ? rq : pk_dkv(a, pk_form(a, dtype, p, 8, Hq), st);
}

}  // extern "C"
