// Argument checks shared by the attention sublayer's entry points.  Host code only.
#pragma once

#include "ssn.h"

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "attn_launch.h"

namespace ssn_checks {

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
inline ssn_status_t heads_ok(int64_t N, int64_t Hq, int64_t Hk, int64_t D, int64_t R, int64_t P, int style,
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
inline bool batch_ok(int64_t N, int64_t B, int64_t Hk, int64_t npages, int64_t page_size, int64_t width) {
  if (B < 0 || B >= kMaxB || N < 0 || N >= kMaxRows || Hk < 1 || npages < 1 || page_size < 1 || width < 1)
    return false;
  return below(width, page_size, kMaxRows) && below(npages, page_size, kMaxRows) &&
         below(npages * page_size, Hk, kMaxRows);
}
inline ssn::PagedBatch paged_batch(int64_t N, int64_t B, int64_t npages, int64_t page_size, const int32_t* pages,
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

// Sizes of an attention over a paged cache.
inline bool attention_shape_ok(int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                               int64_t max_len) {
  return N >= 0 && B >= 0 && B < kMaxB && Hk >= 1 && Hq >= Hk && Hq <= (1 << 20) && Hq % Hk == 0 && D >= 1 &&
         max_q >= 0 && max_q < kMaxRows && max_len >= 0 && max_len < kMaxRows && below(N, Hq, kMaxAttnRows) &&
         below(B, Hk, kMaxAttnSeqs);
}

}  // namespace ssn_checks
