// C ABI of the attention sublayer: argument validation (before any HIP call)
// and dispatch to the kernel launchers.  Contracts: include/ssn.h.
#include "ssn.h"

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "attn_launch.h"

namespace {

constexpr int64_t kMaxElems = (int64_t)1 << 56;   // keeps every byte offset in int64
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 4096;   // rows of heads, cache rows, positions
// Of attention: one grid holds its blocks with one range of keys, and the plan
// takes no more ranges than fit.
constexpr int64_t kMaxAttnRows = (int64_t)1 << 28;
constexpr int64_t kMaxAttnSeqs = (int64_t)1 << 22;         // sequences times key heads
constexpr int64_t kMaxD = 1024;
constexpr int64_t kMaxB = 1 << 20;

inline int64_t elem_size(int dtype) { return dtype == SSN_BF16 ? 2 : 4; }
inline bool valid_dtype(int t) { return t == SSN_F32 || t == SSN_BF16; }
inline bool aligned_to(const void* p, int64_t a) { return ((uintptr_t)p % (uintptr_t)a) == 0; }
inline bool mul_ok(int64_t a, int64_t b) { return a >= 0 && b >= 0 && (a == 0 || b <= kMaxElems / a); }
// a * b below limit, for a, b >= 0
inline bool below(int64_t a, int64_t b, int64_t limit) { return a == 0 || b <= (limit - 1) / a; }
inline ssn_status_t launch_status(hipError_t e) { return e == hipSuccess ? SSN_OK : SSN_ERR_LAUNCH; }

// Memory that a call reads or writes: n rows of w bytes, ld bytes apart.
struct Region {
  uintptr_t p;
  int64_t n, w, ld;
  uintptr_t end() const { return p + (uintptr_t)((n - 1) * ld + w); }
};
inline Region flat(const void* p, int64_t bytes) { return Region{(uintptr_t)p, 1, bytes, bytes}; }
inline Region rows(const void* p, int64_t n, int64_t w, int64_t ld) { return Region{(uintptr_t)p, n, w, ld}; }
// Rows of the same stride overlap where their columns do (parts of one packed
// buffer do not); others if their spans do.
inline bool overlap(const Region& a, const Region& b) {
  if (!a.p || !b.p || a.n < 1 || b.n < 1 || a.w < 1 || b.w < 1) return false;
  if (a.p >= b.end() || b.p >= a.end()) return false;
  if (a.n == 1 || b.n == 1 || a.ld != b.ld) return true;
  const Region &lo = a.p <= b.p ? a : b, &hi = a.p <= b.p ? b : a;
  const int64_t off = (int64_t)((hi.p - lo.p) % (uintptr_t)lo.ld);
  return off < lo.w || off + hi.w > lo.ld;
}
template <int NO, int NI>
inline bool any_overlap(const Region (&out)[NO], const Region (&in)[NI]) {
  for (int i = 0; i < NO; ++i) {
    for (int j = 0; j < NI; ++j)
      if (overlap(out[i], in[j])) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return true;
  }
  return false;
}

// Sizes of heads and rotation, shared by the entry points.
ssn_status_t heads_ok(int64_t N, int64_t Hq, int64_t Hk, int64_t D, int64_t R, int64_t P, int style,
                      float eps, const void* wq, const void* wk) {
  if (N < 0 || Hq < 0 || Hk < 0 || Hq > (1 << 20) || Hk > (1 << 20) || Hq + Hk < 1 || D < 1) return SSN_ERR_SHAPE;
  if (R < 0 || R > D || R % 2 || (R && (P < 1 || P >= kMaxRows))) return SSN_ERR_SHAPE;
  if (style != SSN_ROPE_HALVES && style != SSN_ROPE_PAIRS) return SSN_ERR_SHAPE;
  if (!(eps < INFINITY) || (eps < 0 && (wq || wk))) return SSN_ERR_SHAPE;
  if (!below(N, Hq + 2 * Hk, kMaxRows)) return SSN_ERR_SHAPE;
  return D > kMaxD ? SSN_ERR_UNSUPPORTED : SSN_OK;
}
// Row stride of n rows of H heads.
inline bool ld_ok(int64_t n, int64_t H, int64_t D, int64_t ld) {
  return H == 0 || (ld >= H * D && ld <= kMaxElems && mul_ok(n, ld));
}
inline ssn::HeadRows head_rows(const void* p, int64_t ld, int64_t H) { return ssn::HeadRows{p, ld, (int)H}; }
inline ssn::NormRope norm_rope(int64_t D, int64_t R, int64_t P, int style, float eps, const float* table) {
  return ssn::NormRope{(int)D, (int)R, (int)P, style == SSN_ROPE_PAIRS, eps, table};
}

// Sizes of a paged batch.
bool batch_ok(int64_t N, int64_t B, int64_t Hk, int64_t npages, int64_t page_size, int64_t width) {
  if (B < 0 || B >= kMaxB || N < 0 || N >= kMaxRows || Hk < 1 || npages < 1 || page_size < 1 || width < 1)
    return false;
  return below(width, page_size, kMaxRows) && below(npages, page_size, kMaxRows) &&
         below(npages * page_size, Hk, kMaxRows);
}
ssn::PagedBatch paged_batch(int64_t N, int64_t B, int64_t npages, int64_t page_size, const int32_t* pages,
                            int64_t width, const int32_t* starts, const int32_t* lens, int64_t max_len) {
  ssn::PagedBatch pb;
  pb.pages = pages;
  pb.starts = starts;
  pb.lens = lens;
  pb.width = (int32_t)width;
  pb.npages = (int32_t)npages;
  pb.B = (int32_t)B;
  pb.N = (int32_t)N;
  pb.max_len = (int32_t)(max_len < width * page_size ? max_len : width * page_size);   // < kMaxRows
  pb.page = ssn::fast_div((uint32_t)page_size);
  return pb;
}

}  // namespace

extern "C" {

ssn_status_t ssn_rope_table(int64_t P, int64_t R, double theta, float* table, void* stream) {
  if (P < 0 || P >= kMaxRows || R < 0 || R % 2 || !mul_ok(P, R) || !(theta > 0) || !(theta < INFINITY))
    return SSN_ERR_SHAPE;
  if (P == 0 || R == 0) return SSN_OK;
  if (!table) return SSN_ERR_NULL;
  if (!aligned_to(table, 4)) return SSN_ERR_ALIGN;
  return launch_status(ssn::launch_rope_table(P, R, theta, table, (hipStream_t)stream));
}

ssn_status_t ssn_qk_norm_rope(ssn_dtype_t dtype, int64_t N, int64_t Hq, int64_t Hk, int64_t D, int64_t R,
                              int64_t P, ssn_rope_t style, float eps, const void* Q, int64_t ldq,
                              const void* K, int64_t ldk, const void* wq, const void* wk,
                              const int32_t* pos, const float* table, void* Qout, int64_t ldqo, void* Kout,
                              int64_t ldko, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  if (!Hq) { Q = nullptr; wq = nullptr; Qout = nullptr; ldq = ldqo = 0; }
  if (!Hk) { K = nullptr; wk = nullptr; Kout = nullptr; ldk = ldko = 0; }
  const ssn_status_t st = heads_ok(N, Hq, Hk, D, R, P, style, eps, wq, wk);
  if (st != SSN_OK) return st;
  if (!ld_ok(N, Hq, D, ldq) || !ld_ok(N, Hk, D, ldk) || !ld_ok(N, Hq, D, ldqo) || !ld_ok(N, Hk, D, ldko))
    return SSN_ERR_SHAPE;
  if (N == 0) return SSN_OK;
  if ((Hq && (!Q || !Qout)) || (Hk && (!K || !Kout)) || (R && (!pos || !table))) return SSN_ERR_NULL;
  const int64_t s = elem_size(dtype);
  for (const void* p : {Q, K, (const void*)Qout, (const void*)Kout, wq, wk})
    if (!aligned_to(p, s)) return SSN_ERR_ALIGN;
  if (R && (!aligned_to(pos, 4) || !aligned_to(table, 4))) return SSN_ERR_ALIGN;
  const Region out[] = {rows(Qout, N, Hq * D * s, ldqo * s), rows(Kout, N, Hk * D * s, ldko * s)};
  const Region in[] = {rows(Q, N, Hq * D * s, ldq * s), rows(K, N, Hk * D * s, ldk * s), flat(wq, D * s),
                       flat(wk, D * s), flat(R ? pos : nullptr, N * 4), flat(R ? table : nullptr, P * R * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  return launch_status(ssn::launch_norm_rope(dtype, N, norm_rope(D, R, P, style, eps, table),
                                             head_rows(Q, ldq, Hq), head_rows(K, ldk, Hk), wq, wk, pos,
                                             head_rows(Qout, ldqo, Hq), head_rows(Kout, ldko, Hk),
                                             (hipStream_t)stream));
}

size_t ssn_qk_norm_rope_workspace_bytes(ssn_dtype_t dtype, int64_t N, int64_t Hq, int64_t Hk, int64_t D) {
  if (!valid_dtype(dtype) || heads_ok(N, Hq, Hk, D, 0, 1, SSN_ROPE_HALVES, 0.f, nullptr, nullptr) != SSN_OK ||
      N == 0)
    return 0;
  return (size_t)ssn::norm_rope_backward_blocks(N, Hq + Hk) * 2 * (size_t)D * 4;
}

ssn_status_t ssn_qk_norm_rope_backward(ssn_dtype_t dtype, int64_t N, int64_t Hq, int64_t Hk, int64_t D,
                                       int64_t R, int64_t P, ssn_rope_t style, float eps, const void* Q,
                                       int64_t ldq, const void* K, int64_t ldk, const void* wq,
                                       const void* wk, const int32_t* pos, const float* table,
                                       const void* GQ, int64_t ldgq, const void* GK, int64_t ldgk,
                                       void* GQin, int64_t ldgqi, void* GKin, int64_t ldgki, float* Gwq,
                                       float* Gwk, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  if (!Hq) { Q = nullptr; wq = nullptr; GQ = nullptr; GQin = nullptr; ldq = ldgq = ldgqi = 0; }
  if (!Hk) { K = nullptr; wk = nullptr; GK = nullptr; GKin = nullptr; ldk = ldgk = ldgki = 0; }
  const ssn_status_t st = heads_ok(N, Hq, Hk, D, R, P, style, eps, wq, wk);
  if (st != SSN_OK) return st;
  if (!ld_ok(N, Hq, D, ldq) || !ld_ok(N, Hk, D, ldk) || !ld_ok(N, Hq, D, ldgq) || !ld_ok(N, Hk, D, ldgk) ||
      !ld_ok(N, Hq, D, ldgqi) || !ld_ok(N, Hk, D, ldgki))
    return SSN_ERR_SHAPE;
  if (eps < 0 && (Gwq || Gwk)) return SSN_ERR_SHAPE;
  const bool wants = Gwq || Gwk;
  const int64_t need = wants ? (int64_t)ssn_qk_norm_rope_workspace_bytes(dtype, N, Hq, Hk, D) : 0;
  if (N == 0 && !wants) return SSN_OK;
  const int64_t s = elem_size(dtype);
  if (N > 0) {
    if ((Hq && (!Q || !GQ || !GQin)) || (Hk && (!K || !GK || !GKin)) || (R && (!pos || !table)) ||
        (need && !workspace))
      return SSN_ERR_NULL;
    if (workspace_bytes < (size_t)need) return SSN_ERR_SHAPE;
    for (const void* p : {Q, K, wq, wk, GQ, GK, (const void*)GQin, (const void*)GKin})
      if (!aligned_to(p, s)) return SSN_ERR_ALIGN;
    if (R && (!aligned_to(pos, 4) || !aligned_to(table, 4))) return SSN_ERR_ALIGN;
  }
  if (!aligned_to(Gwq, 4) || !aligned_to(Gwk, 4) || (need && !aligned_to(workspace, 4))) return SSN_ERR_ALIGN;
  const Region out[] = {rows(GQin, N, Hq * D * s, ldgqi * s), rows(GKin, N, Hk * D * s, ldgki * s),
                        flat(Gwq, D * 4), flat(Gwk, D * 4), flat(need ? workspace : nullptr, need)};
  const Region in[] = {rows(Q, N, Hq * D * s, ldq * s),   rows(K, N, Hk * D * s, ldk * s),
                       rows(GQ, N, Hq * D * s, ldgq * s), rows(GK, N, Hk * D * s, ldgk * s),
                       flat(wq, D * s),                   flat(wk, D * s),
                       flat(R ? pos : nullptr, N * 4),    flat(R ? table : nullptr, P * R * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  return launch_status(ssn::launch_norm_rope_backward(
      dtype, N, norm_rope(D, R, P, style, eps, table), head_rows(Q, ldq, Hq), head_rows(K, ldk, Hk), wq, wk,
      pos, head_rows(GQ, ldgq, Hq), head_rows(GK, ldgk, Hk), head_rows(GQin, ldgqi, Hq),
      head_rows(GKin, ldgki, Hk), Gwq, Gwk, (float*)workspace, (hipStream_t)stream));
}

ssn_status_t ssn_kv_append(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                           int64_t R, int64_t P, ssn_rope_t style, float eps, const void* Q, int64_t ldq,
                           const void* K, int64_t ldk, const void* V, int64_t ldv, const void* wq,
                           const void* wk, const float* table, void* Kc, void* Vc, int64_t npages,
                           int64_t page_size, const int32_t* pages, int64_t width, const int32_t* starts,
                           const int32_t* lens, void* Qout, int64_t ldqo, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  if (!Hq) { Q = nullptr; wq = nullptr; Qout = nullptr; ldq = ldqo = 0; }
  const ssn_status_t st = heads_ok(N, Hq, Hk, D, R, P, style, eps, wq, wk);
  if (st != SSN_OK) return st;
  if (!batch_ok(N, B, Hk, npages, page_size, width) || !mul_ok(npages * page_size * Hk, D)) return SSN_ERR_SHAPE;
  if (!ld_ok(N, Hq, D, ldq) || !ld_ok(N, Hk, D, ldk) || !ld_ok(N, Hk, D, ldv) || !ld_ok(N, Hq, D, ldqo))
    return SSN_ERR_SHAPE;
  if (N == 0 || B == 0) return SSN_OK;
  if ((Hq && (!Q || !Qout)) || !K || !V || !Kc || !Vc || !pages || !starts || !lens || (R && !table))
    return SSN_ERR_NULL;
  const int64_t s = elem_size(dtype);
  for (const void* p : {Q, K, V, wq, wk, (const void*)Kc, (const void*)Vc, (const void*)Qout})
    if (!aligned_to(p, s)) return SSN_ERR_ALIGN;
  if (!aligned_to(pages, 4) || !aligned_to(starts, 4) || !aligned_to(lens, 4) || (R && !aligned_to(table, 4)))
    return SSN_ERR_ALIGN;
  const int64_t cache = npages * page_size * Hk * D * s;
  const Region out[] = {rows(Qout, N, Hq * D * s, ldqo * s), flat(Kc, cache), flat(Vc, cache)};
  const Region in[] = {rows(Q, N, Hq * D * s, ldq * s), rows(K, N, Hk * D * s, ldk * s),
                       rows(V, N, Hk * D * s, ldv * s), flat(wq, D * s), flat(wk, D * s),
                       flat(R ? table : nullptr, P * R * 4), flat(pages, B * width * 4),
                       flat(starts, (B + 1) * 4), flat(lens, B * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  return launch_status(ssn::launch_kv_append(
      dtype, paged_batch(N, B, npages, page_size, pages, width, starts, lens, kMaxRows),
      norm_rope(D, R, P, style, eps, table), head_rows(Q, ldq, Hq), head_rows(K, ldk, Hk),
      head_rows(V, ldv, Hk), wq, wk, Kc, Vc, head_rows(Qout, ldqo, Hq), (hipStream_t)stream));
}

static bool attention_shape_ok(int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                               int64_t max_len) {
  return N >= 0 && B >= 0 && B < kMaxB && Hk >= 1 && Hq >= Hk && Hq <= (1 << 20) && Hq % Hk == 0 && D >= 1 &&
         max_q >= 0 && max_q < kMaxRows && max_len >= 0 && max_len < kMaxRows && below(N, Hq, kMaxAttnRows) &&
         below(B, Hk, kMaxAttnSeqs);
}

size_t ssn_paged_attention_workspace_bytes(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk,
                                           int64_t D, int64_t max_q, int64_t max_len) {
  if (!valid_dtype(dtype) || !attention_shape_ok(N, B, Hq, Hk, D, max_q, max_len) || D > kMaxD || N == 0 ||
      B == 0)
    return 0;
  return ssn::attention_workspace_bytes(dtype, N, B, Hq, Hk, D, max_q, max_len);
}

ssn_status_t ssn_paged_attention(ssn_dtype_t dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                                 int64_t max_q, int64_t max_len, float scale, const void* Q, int64_t ldq,
                                 const void* Kc, const void* Vc, int64_t npages, int64_t page_size,
                                 const int32_t* pages, int64_t width, const int32_t* starts,
                                 const int32_t* lens, void* O, int64_t ldo, float* lse, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  if (!valid_dtype(dtype)) return SSN_ERR_DTYPE;
  if (!attention_shape_ok(N, B, Hq, Hk, D, max_q, max_len) ||
      !batch_ok(N, B, Hk, npages, page_size, width))
    return SSN_ERR_SHAPE;
  if (D > kMaxD) return SSN_ERR_UNSUPPORTED;
  if (!mul_ok(npages * page_size * Hk, D) ||
      !(scale > -INFINITY && scale < INFINITY) || !ld_ok(N, Hq, D, ldq) || !ld_ok(N, Hq, D, ldo))
    return SSN_ERR_SHAPE;
  if (N == 0 || B == 0) return SSN_OK;
  if (!Q || !Kc || !Vc || !pages || !starts || !lens || !O || (workspace_bytes && !workspace))
    return SSN_ERR_NULL;
  const int64_t s = elem_size(dtype);
  for (const void* p : {Q, Kc, Vc, (const void*)O})
    if (!aligned_to(p, s)) return SSN_ERR_ALIGN;
  if (!aligned_to(pages, 4) || !aligned_to(starts, 4) || !aligned_to(lens, 4) || !aligned_to(lse, 4) ||
      (workspace_bytes && !aligned_to(workspace, 16)))
    return SSN_ERR_ALIGN;
  if (workspace_bytes > UINTPTR_MAX - (uintptr_t)workspace || workspace_bytes > (size_t)INT64_MAX)
    return SSN_ERR_SHAPE;
  const int64_t cache = npages * page_size * Hk * D * s;
  const Region out[] = {rows(O, N, Hq * D * s, ldo * s), flat(lse, N * Hq * 4),
                        flat(workspace_bytes ? workspace : nullptr, (int64_t)workspace_bytes)};
  const Region in[] = {rows(Q, N, Hq * D * s, ldq * s), flat(Kc, cache), flat(Vc, cache),
                       flat(pages, B * width * 4), flat(starts, (B + 1) * 4), flat(lens, B * 4)};
  if (any_overlap(out, in)) return SSN_ERR_ALIAS;
  ssn::AttnArgs a;
  a.pb = paged_batch(N, B, npages, page_size, pages, width, starts, lens, max_len);
  a.Q = Q;
  a.Kc = Kc;
  a.Vc = Vc;
  a.O = O;
  a.lse = lse;
  a.ldq = ldq;
  a.ldo = ldo;
  a.Hq = (int)Hq;
  a.Hk = (int)Hk;
  a.D = (int)D;
  a.G = (int)(Hq / Hk);
  a.max_q = (int)max_q;
  a.scale = scale;
  return launch_status(ssn::launch_paged_attention(dtype, a, workspace, workspace_bytes, (hipStream_t)stream));
}

}  // extern "C"
