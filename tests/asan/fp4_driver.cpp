// Drives the 4-bit cache's host-side validation with ordinary, edge and hostile
// sizes under AddressSanitizer and UndefinedBehaviorSanitizer.  The launchers are
// stubs that check what they are given: a call that reaches one has sizes that
// fit the kernels' 32-bit indices.
#include <stdint.h>
#include <stdio.h>

#include "fp4_launch.h"
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
static void batch_fits(const PagedBatch& b, int D) {
  expect(b.B > 0 && b.N > 0 && b.npages > 0 && b.width > 0 && b.page.d > 0, "batch sizes");
  expect((int64_t)b.width * b.page.d < ((int64_t)1 << 31) && b.max_len <= (int64_t)b.width * b.page.d, "positions");
  expect(D > 0 && D % kFp4Group == 0 && D <= 1024, "head size");
}

hipError_t launch_kv_append_fp4(int, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k, HeadRows v,
                                const void*, const void*, const Fp4Cache& c, HeadRows qo, hipStream_t) {
  for (const HeadRows& r : {q, k, v, qo}) heads_fit(r, nr.D);
  batch_fits(pb, nr.D);
  expect(c.Kc && c.Ks && c.Vc && c.Vs, "cache");
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_kv_read_fp4(int, const PagedBatch& pb, int D, const Fp4Cache& c, HeadRows k, HeadRows v,
                              hipStream_t) {
  for (const HeadRows& r : {k, v}) heads_fit(r, D);
  batch_fits(pb, D);
  expect(c.Kc && c.Ks && c.Vc && c.Vs, "cache");
  ++g_launches;
  return hipSuccess;
}
size_t fp4_attention_workspace_bytes(int, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return 64; }
hipError_t launch_paged_attention_fp4(int, const Fp4AttnArgs& f, void*, size_t, hipStream_t) {
  batch_fits(f.a.pb, f.a.D);
  expect(f.a.Hq == f.a.G * f.a.Hk && (int64_t)f.a.pb.N * f.a.Hq < ((int64_t)1 << 31), "heads");
  expect(f.a.Kc && f.Ks && f.a.Vc && f.Vs, "cache");
  ++g_launches;
  return hipSuccess;
}

}  // namespace ssn

int main() {
  auto P = [](uint64_t i) { return (void*)(i << 44); };
  auto U = [](uint64_t i) { return (uint8_t*)(i << 44); };
  const int64_t big = INT64_MAX;
  const int64_t sizes[] = {-big - 1, -1, 0, 1, 2, 32, 64, 96, 1000, (int64_t)1 << 20, (int64_t)1 << 31,
                           (int64_t)1 << 40, (int64_t)1 << 56, big};
  for (int64_t N : sizes)
    for (int64_t H : sizes)
      for (int64_t D : sizes)
        for (int64_t ld : sizes) {
          ssn_paged_attention_fp4_workspace_bytes(SSN_BF16, N, H, H, H, D, ld, N);
          for (int64_t pages : {(int64_t)1, (int64_t)1000, (int64_t)1 << 31, big})
            for (int64_t size : {(int64_t)0, (int64_t)1, (int64_t)16, (int64_t)1 << 20, big}) {
              ssn_kv_append_fp4(SSN_BF16, N, 3, H, 2, D, 0, 1, SSN_ROPE_HALVES, -1.f, P(1), ld, P(2), ld, P(3), ld,
                                nullptr, nullptr, nullptr, U(4), U(5), U(10), U(11), pages, size, (int32_t*)P(6),
                                pages, (int32_t*)P(7), (int32_t*)P(8), P(9), ld, nullptr);
              ssn_kv_read_fp4(SSN_F32, N, 3, H, D, U(4), U(5), U(10), U(11), pages, size, (int32_t*)P(6), 17,
                              (int32_t*)P(7), (int32_t*)P(8), P(1), ld, P(2), ld, nullptr);
              ssn_paged_attention_fp4(SSN_F32, N, 3, H, 1, D, N, ld, 1.f, P(1), ld, U(2), U(3), U(10), U(11), pages,
                                      size, (int32_t*)P(4), 17, (int32_t*)P(5), (int32_t*)P(6), P(7), ld,
                                      (float*)P(8), P(9), (size_t)1 << 30, nullptr);
            }
        }
  expect(g_launches > 0, "no call reached a launcher");
  if (g_fail) return 1;
  printf("4-bit cache validation ok (%ld launches)\n", g_launches);
  return 0;
}
