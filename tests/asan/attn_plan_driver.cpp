// The attention's plan (kernels, tiles, ranges of keys, workspace) over the sizes
// that its entry point lets through, under UndefinedBehaviorSanitizer.
#include <stdint.h>
#include <stdio.h>

#include "attn_plan.h"

static long g_fail = 0;
static void expect(bool ok, const char* what, int64_t N, int64_t B, int64_t Hk, int64_t max_q, int64_t max_len) {
  if (ok) return;
  if (++g_fail < 10)
    fprintf(stderr, "%s: N=%lld B=%lld Hk=%lld max_q=%lld max_len=%lld\n", what, (long long)N, (long long)B,
            (long long)Hk, (long long)max_q, (long long)max_len);
}

int main() {
  long cases = 0;
  for (int dtype : {0, 1})
    for (int64_t D : {8, 64, 128, 256})
      for (int64_t Hk : {1, 2, 8, 40, 1000, 65536, 1 << 20})
        for (int64_t G : {1, 2, 5, 16, 17, 1024}) {
          const int64_t Hq = Hk * G;
          if (Hq > (1 << 20)) continue;
          for (int64_t N : {1, 2, 63, 200, 519, 4096, 100000, 1 << 20, 1 << 24, (1 << 28) - 1}) {
            if (N * Hq >= (int64_t)1 << 28) continue;
            for (int64_t B : {1, 2, 3, 64, 257, 10000, 100000, 200000, (1 << 20) - 1}) {
              if (B * Hk >= (int64_t)1 << 22) continue;
              for (int64_t max_q : {0, 1, 2, 4, 17, 64, 517, 100000, 2147479551})
                for (int64_t max_len : {0, 1, 100, 2000, 8191, 8192, 40000, 131072, 2147479551})
                  for (uint64_t ws : {(uint64_t)0, (uint64_t)1000, (uint64_t)(1 << 20) + 8, (uint64_t)1 << 60}) {
                    const ssn::AttnPlan p = ssn::attention_plan(dtype, N, B, Hq, Hk, D, max_q, max_len, ws);
                    const int64_t tiles = ssn::tile_blocks(p, N, B, Hk, G), rows = ssn::row_blocks(p, B, Hk);
#define CHECK(x) expect(x, #x, N, B, Hk, max_q, max_len)
                    CHECK(tiles + rows > 0 && tiles + rows < (int64_t)1 << 24);
                    CHECK(tiles == 0 || tiles >= ssn::tile_slots(N, B, G, 64 * p.tiles.blocks) * Hk);
                    const uint64_t at = ssn::stage_bytes(p.tiles, D), end = at + ssn::stage_bytes(p.rows, D);
                    CHECK(at % 16 == 0 && end % 16 == 0 && end <= ws);
                    for (const ssn::AttnPart* x : {&p.tiles, &p.rows}) {
                      if (!x->blocks) continue;
                      CHECK(x->ranges >= 1 && x->ranges <= ssn::kMaxRanges);
                      CHECK(x->chunk > 0 && x->chunk % 128 == 0 && (int64_t)x->chunk * x->ranges >= max_len);
                      CHECK(ssn::key_ranges((int)(max_len > 1 ? max_len : 1), x->chunk) == x->ranges);
                    }
                    ++cases;
                  }
            }
          }
        }
  if (g_fail) {
    fprintf(stderr, "%ld of %ld failed\n", g_fail, cases);
    return 1;
  }
  printf("attention plans ok (%ld cases)\n", cases);
  return 0;
}
