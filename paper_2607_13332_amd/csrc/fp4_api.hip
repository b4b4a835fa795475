// C ABI of the 4-bit cache: argument validation (before any HIP call) and
// dispatch to the kernel launchers.  Contracts: include/ssn.h.
#include "attn_checks.h"
#include "fp4_launch.h"

using namespace ssn_checks;

namespace {

struct CacheBytes {
  int64_t codes, scales;
};
// Heads of D elements in groups of 32, and a cache whose bytes fit.
bool fp4_cache_ok(int64_t npages, int64_t page_size, int64_t Hk, int64_t D, CacheBytes& n) {
  if (D < 1 || D % ssn::kFp4Group || !mul_ok(npages * page_size * Hk, D)) return false;
  const int64_t heads = npages * page_size * Hk;
  n = CacheBytes{heads * (D / 2), heads * (D / ssn::kFp4Group)};
  return true;
}

}  // namespace

extern "C" {

ssn_status_t ssn_kv_append_fp4(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                               int64_t R, int64_t P, ssn_rope_t style, float eps, const void* Q, int64_t ldq,
                               const void* K, int64_t ldk, const void* V, int64_t ldv, const void* wq,
                               const void* wk, const float* table, uint8_t* Kc, uint8_t* Ks, uint8_t* Vc,
                               uint8_t* Vs, int64_t npages, int64_t page_size, const int32_t* pages,
                               int64_t width, const int32_t* starts, const int32_t* lens, void* Qout,
                               int64_t ldqo, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  if (!Hq) { Q = nullptr; wq = nullptr; Qout = nullptr; ldq = ldqo = 0; }
  const ssn_status_t st = heads_ok(N, Hq, Hk, D, R, P, style, eps, wq, wk);
  if (st != SSN_OK) return st;
  CacheBytes n;
  if (!batch_ok(N, B, Hk, npages, page_size, width) || !fp4_cache_ok(npages, page_size, Hk, D, n))
    return SSN_ERR_SHAPE;
  if (!ld_ok(N, Hq, D, ldq) || !ld_ok(N, Hk, D, ldk) || !ld_ok(N, Hk, D, ldv) || !ld_ok(N, Hq, D, ldqo))
    return SSN_ERR_SHAPE;
  if (N == 0 || B == 0) return SSN_OK;
  if ((Hq && (!Q || !Qout)) || !K || !V || !Kc || !Ks || !Vc || !Vs || !pages || !starts || !lens || (R && !table))
    return SSN_ERR_NULL;
  const int64_t s = elem_size(dtype);
  for (const void* p : {Q, K, V, wq, wk, (const void*)Qout})
    if (!aligned_to(p, s)) return SSN_ERR_ALIGN;
  if (!aligned_to(pages, 4) || !aligned_to(starts, 4) || !aligned_to(lens, 4) || (R && !aligned_to(table, 4)))
    return SSN_ERR_ALIGN;
  const Region out[] = {rows(Qout, N, Hq * D * s, ldqo * s), flat(Kc, n.codes), flat(Ks, n.scales),
                        flat(Vc, n.codes), flat(Vs, n.scales)};
  const Region in[] = {rows(Q, N, Hq * D * s, ldq * s), rows(K, N, Hk * D * s, ldk * s),
                       rows(V, N, Hk * D * s, ldv * s), flat(wq, D * s), flat(wk, D * s),
                       flat(R ? table : nullptr, P * R * 4), flat(pages, B * width * 4),
                       flat(starts, (B + 1) * 4), flat(lens, B * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  return launch_status(ssn::launch_kv_append_fp4(
      dtype, paged_batch(N, B, npages, page_size, pages, width, starts, lens, kMaxRows),
      norm_rope(D, R, P, style, eps, table), head_rows(Q, ldq, Hq), head_rows(K, ldk, Hk),
      head_rows(V, ldv, Hk), wq, wk, ssn::Fp4Cache{Kc, Ks, Vc, Vs}, head_rows(Qout, ldqo, Hq),
      (hipStream_t)stream));
}

ssn_status_t ssn_kv_read_fp4(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hk, int64_t D, const uint8_t* Kc,
                             const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs, int64_t npages,
                             int64_t page_size, const int32_t* pages, int64_t width, const int32_t* starts,
                             const int32_t* lens, void* K, int64_t ldk, void* V, int64_t ldv, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  const ssn_status_t st = heads_ok(N, 0, Hk, D, 0, 1, SSN_ROPE_HALVES, -1.f, nullptr, nullptr);
  if (st != SSN_OK) return st;
  CacheBytes n;
  if (!batch_ok(N, B, Hk, npages, page_size, width) || !fp4_cache_ok(npages, page_size, Hk, D, n) ||
      !ld_ok(N, Hk, D, ldk) || !ld_ok(N, Hk, D, ldv))
    return SSN_ERR_SHAPE;
  if (N == 0 || B == 0) return SSN_OK;
  if (!Kc || !Ks || !Vc || !Vs || !pages || !starts || !lens || !K || !V) return SSN_ERR_NULL;
  const int64_t s = elem_size(dtype);
  if (!aligned_to(K, s) || !aligned_to(V, s) || !aligned_to(pages, 4) || !aligned_to(starts, 4) ||
      !aligned_to(lens, 4))
    return SSN_ERR_ALIGN;
  const Region out[] = {rows(K, N, Hk * D * s, ldk * s), rows(V, N, Hk * D * s, ldv * s)};
  const Region in[] = {flat(Kc, n.codes), flat(Ks, n.scales), flat(Vc, n.codes), flat(Vs, n.scales),
                       flat(pages, B * width * 4), flat(starts, (B + 1) * 4), flat(lens, B * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  return launch_status(ssn::launch_kv_read_fp4(
      dtype, paged_batch(N, B, npages, page_size, pages, width, starts, lens, kMaxRows), (int)D,
      ssn::Fp4Cache{(uint8_t*)Kc, (uint8_t*)Ks, (uint8_t*)Vc, (uint8_t*)Vs}, head_rows(K, ldk, Hk),
      head_rows(V, ldv, Hk), (hipStream_t)stream));
}

size_t ssn_paged_attention_fp4_workspace_bytes(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk,
                                               int64_t D, int64_t max_q, int64_t max_len) {
  if (!valid_dtype(dtype) || !attention_shape_ok(N, B, Hq, Hk, D, max_q, max_len) || D % ssn::kFp4Group ||
      D > kMaxD || N == 0 || B == 0)
    return 0;
  return ssn::fp4_attention_workspace_bytes(dtype, N, B, Hq, Hk, D, max_q, max_len);
}

ssn_status_t ssn_paged_attention_fp4(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                                     int64_t max_q, int64_t max_len, float scale, const void* Q, int64_t ldq,
                                     const uint8_t* Kc, const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs,
                                     int64_t npages, int64_t page_size, const int32_t* pages, int64_t width,
                                     const int32_t* starts, const int32_t* lens, void* O, int64_t ldo, float* lse,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  if (!attention_shape_ok(N, B, Hq, Hk, D, max_q, max_len) || D % ssn::kFp4Group ||
      !batch_ok(N, B, Hk, npages, page_size, width))
    return SSN_ERR_SHAPE;
  if (D > kMaxD) return SSN_ERR_UNSUPPORTED;
  CacheBytes n;
  if (!fp4_cache_ok(npages, page_size, Hk, D, n) || !(scale > -INFINITY && scale < INFINITY) ||
      !ld_ok(N, Hq, D, ldq) || !ld_ok(N, Hq, D, ldo))
    return SSN_ERR_SHAPE;
  if (N == 0 || B == 0) return SSN_OK;
  if (!Q || !Kc || !Ks || !Vc || !Vs || !pages || !starts || !lens || !O || (workspace_bytes && !workspace))
    return SSN_ERR_NULL;
  const int64_t s = elem_size(dtype);
  if (!aligned_to(Q, s) || !aligned_to(O, s) || !aligned_to(pages, 4) || !aligned_to(starts, 4) ||
      !aligned_to(lens, 4) || !aligned_to(lse, 4) || (workspace_bytes && !aligned_to(workspace, 16)))
    return SSN_ERR_ALIGN;
  if (workspace_bytes > UINTPTR_MAX - (uintptr_t)workspace || workspace_bytes > (size_t)INT64_MAX)
    return SSN_ERR_SHAPE;
  const Region out[] = {rows(O, N, Hq * D * s, ldo * s), flat(lse, N * Hq * 4),
                        flat(workspace_bytes ? workspace : nullptr, (int64_t)workspace_bytes)};
  const Region in[] = {rows(Q, N, Hq * D * s, ldq * s), flat(Kc, n.codes), flat(Ks, n.scales),
                       flat(Vc, n.codes), flat(Vs, n.scales), flat(pages, B * width * 4),
                       flat(starts, (B + 1) * 4), flat(lens, B * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  ssn::Fp4AttnArgs f;
  f.a.pb = paged_batch(N, B, npages, page_size, pages, width, starts, lens, max_len);
  f.a.Q = Q;
  f.a.Kc = Kc;
  f.a.Vc = Vc;
  f.a.O = O;
  f.a.lse = lse;
  f.a.ldq = ldq;
  f.a.ldo = ldo;
  f.a.Hq = (int)Hq;
  f.a.Hk = (int)Hk;
  f.a.D = (int)D;
  f.a.G = (int)(Hq / Hk);
  f.a.max_q = (int)max_q;
  f.a.scale = scale;
  f.Ks = Ks;
  f.Vs = Vs;
  return launch_status(ssn::launch_paged_attention_fp4(dtype, f, workspace, workspace_bytes, (hipStream_t)stream));
}

}  // extern "C"
