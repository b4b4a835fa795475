// Drives the attention sublayer's host-side validation with ordinary, edge
// and hostile sizes under AddressSanitizer and UndefinedBehaviorSanitizer.
// The launchers are stubs that check what they are given: a call that reaches
// one has sizes that fit the kernels' 32-bit indices.
#include <stdint.h>
#include <stdio.h>

#include "attn_launch.h"
#include "ssn.h"

static long g_launches = 0, g_fail = 0;

static void expect(bool ok, const char* what) {
  if (!ok) {
    fprintf(stderr, "unexpected: %s\n", what);
    ++g_fail;
  }
}

namespace ssn {

static void heads_fit(const HeadRows& r, int D) { expect(r.H == 0 || (r.p && r.ld >= (int64_t)r.H * D), "row stride"); }
static void batch_fits(const PagedBatch& b) {
  expect(b.B > 0 && b.N > 0 && b.npages > 0 && b.width > 0 && b.page.d > 0, "batch sizes");
  expect((int64_t)b.width * b.page.d < ((int64_t)1 << 31) && b.max_len <= (int64_t)b.width * b.page.d, "positions");
  // the multiplication is exact at both ends of every quotient
  for (uint64_t x : {(uint64_t)0, (uint64_t)1, (uint64_t)b.page.d - 1, (uint64_t)b.page.d, (uint64_t)b.page.d * 2 - 1,
                     (uint64_t)0x7FFFFFFF, (uint64_t)0x7FFFFFFF / b.page.d * b.page.d})
    expect(x > 0x7FFFFFFF || ((x * b.page.m) >> (31 + b.page.s)) == x / b.page.d, "division");
}

hipError_t launch_rope_table(int64_t, int64_t, double, float*, hipStream_t) {
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_norm_rope(int, int64_t N, const NormRope& nr, HeadRows q, HeadRows k, const void*, const void*,
                            const int32_t*, HeadRows qo, HeadRows ko, hipStream_t) {
  for (const HeadRows& r : {q, k, qo, ko}) heads_fit(r, nr.D);
  expect(N > 0 && nr.R <= nr.D && nr.D <= 1024, "norm sizes");
  ++g_launches;
  return hipSuccess;
}
int norm_rope_backward_blocks(int64_t N, int64_t heads) { return N * heads > 1000 ? 2048 : 1; }
hipError_t launch_norm_rope_backward(int, int64_t, const NormRope& nr, HeadRows q, HeadRows k, const void*,
                                     const void*, const int32_t*, HeadRows gq, HeadRows gk, HeadRows, HeadRows,
                                     float*, float*, float*, hipStream_t) {
  expect(nr.D <= 1024 && q.H == gq.H && k.H == gk.H, "backward sizes");
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_kv_append(int, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k, HeadRows v,
                            const void*, const void*, void*, void*, HeadRows qo, hipStream_t) {
  for (const HeadRows& r : {q, k, v, qo}) heads_fit(r, nr.D);
  batch_fits(pb);
  ++g_launches;
  return hipSuccess;
}
size_t attention_workspace_bytes(int, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return 64; }
hipError_t launch_paged_attention(int, const AttnArgs& a, void*, size_t, hipStream_t) {
  batch_fits(a.pb);
  expect(a.Hq == a.G * a.Hk && (int64_t)a.pb.N * a.Hq < ((int64_t)1 << 31), "heads");
  ++g_launches;
  return hipSuccess;
}

}  // namespace ssn

int main() {
  auto P = [](uint64_t i) { return (void*)(i << 44); };
  const int64_t big = INT64_MAX;
  const int64_t sizes[] = {-big - 1, -1, 0, 1, 2, 7, 64, 1000, (int64_t)1 << 20, (int64_t)1 << 31, (int64_t)1 << 40,
                           (int64_t)1 << 56, big};
  for (int64_t N : sizes)
    for (int64_t Hq : sizes)
      for (int64_t D : sizes)
        for (int64_t ld : sizes) {
          for (int64_t Hk : {(int64_t)0, (int64_t)1, (int64_t)4, big}) {
            for (int64_t R : {(int64_t)0, (int64_t)2, (int64_t)64, big - 1}) {
              ssn_qk_norm_rope(SSN_BF16, N, Hq, Hk, D, R, 100, SSN_ROPE_HALVES, 1e-6f, P(1), ld, P(2), ld, P(3), P(4),
                               (int32_t*)P(5), (float*)P(6), P(7), ld, P(8), ld, nullptr);
              ssn_qk_norm_rope_backward(SSN_F32, N, Hq, Hk, D, R, 100, SSN_ROPE_PAIRS, 1e-6f, P(1), ld, P(2), ld, P(3),
                                        P(4), (int32_t*)P(5), (float*)P(6), P(7), ld, P(8), ld, P(9), ld, P(10), ld,
                                        (float*)P(11), (float*)P(12), P(13), (size_t)1 << 40, nullptr);
            }
            ssn_qk_norm_rope_workspace_bytes(SSN_BF16, N, Hq, Hk, D);
            ssn_paged_attention_workspace_bytes(SSN_BF16, N, Hk, Hq, Hk, D, ld, N);
          }
          for (int64_t pages : {(int64_t)1, (int64_t)1000, (int64_t)1 << 31, big})
            for (int64_t size : {(int64_t)0, (int64_t)1, (int64_t)3, (int64_t)16, (int64_t)1 << 20, big}) {
              ssn_kv_append(SSN_BF16, N, 3, Hq, 2, D, 0, 1, SSN_ROPE_HALVES, -1.f, P(1), ld, P(2), ld, P(3), ld,
                            nullptr, nullptr, nullptr, P(4), P(5), pages, size, (int32_t*)P(6), pages,
                            (int32_t*)P(7), (int32_t*)P(8), P(9), ld, nullptr);
              ssn_paged_attention(SSN_F32, N, 3, Hq, 1, D, N, ld, 1.f, P(1), ld, P(2), P(3), pages, size,
                                  (int32_t*)P(4), 17, (int32_t*)P(5), (int32_t*)P(6), P(7), ld, (float*)P(8), P(9),
                                  (size_t)1 << 30, nullptr);
            }
        }
  for (int64_t p : sizes)
    for (int64_t r : sizes) ssn_rope_table(p, r, 1e4, (float*)P(1), nullptr);
  // every page size's division, at the quotients' ends
  for (uint32_t d = 1; d < 70000; d += d < 300 ? 1 : 997) {
    const ssn::FastDiv f = ssn::fast_div(d);
    for (uint64_t k = 0; k * d <= 0x7FFFFFFF; k += 1 + k / 3)
      for (uint64_t x : {k * d, k * d + d - 1})
        if (x <= 0x7FFFFFFF) expect(((x * f.m) >> (31 + f.s)) == x / d, "fast_div");
  }
  expect(g_launches > 0, "no call reached a launcher");
  if (g_fail) return 1;
  printf("attention validation ok (%ld launches)\n", g_launches);
  return 0;
}
