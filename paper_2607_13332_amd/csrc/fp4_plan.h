// How an attention call over a 4-bit cache is run: attn_plan.h's plan, tuned for a
// quarter of the bytes.  Host code only.
#pragma once

#include "attn_plan.h"

namespace ssn {

// Rows kernel: a block's four waves take 128 keys at a time, and a range of fewer than
// 256 is mostly the wait for its first.  64 single tokens over caches of 1 to 4096
// keys (8 heads of 128) take 47 / 43 / 43 / 43 us for 512 / 1024 / 1536 / 2048 blocks,
// 16 over up to 8192 32 / 26 / 30 / 31.  Ranges cost their join, 4 us and more, which
// shorter ones do not give back where the pairs fill the chip by themselves: 64
// sequences of up to 512 / 1024 / 2048 / 4096 keys take 12 / 16 / 27 / 48 us with one
// range each and 20 / 24 / 33 / 44 with ranges for 1024 blocks.
//
// Beside the rows' blocks tiles do not need the whole chip: 517 tokens and 31 single
// ones over up to 8192 keys take 150 / 121 / 125 us with 256 / 384 / 512 blocks, 256
// tokens and 63 over up to 4096 87 / 90 / 97, 200 tokens and 15 over up to 32768 195 /
// 195 / 207.
//
// Tiles: as wide as fills the chip, us for 64 / 128 / 192 rows: one prompt of 1024 tokens
// (40 / 8 heads of 128) 27 / 32 / 48, 2048 77 / 57 / 75, 4096 252 / 179 / 162; of heads of
// 64 (32 / 8) 2048 33 / 39, 4096 101 / 88.  Chunks at the end of much longer sequences
// have their keys split to fill it: 64 tokens over 8000 keys 37 / 34 / 35, 256 80 / 75 /
// 65, twice 512 over 6000 150 / 139 / 151 (the rule takes 192 rows there too: it does not
// look at how many of the chip's places a width leaves empty).
inline int fp4_tile_rows(int dtype, int64_t rows, int64_t most, int64_t max_q, int64_t Hk, int64_t D,
                         int64_t max_len) {
  if (dtype != kBF16 || D > 128 || most <= 64) return 1;
  const bool split = max_len >= 8192 || max_len / 8 >= max_q;
  if (D <= 64) return split || rows * Hk / 128 >= 768 ? 2 : 1;
  if (most > 128 && (split || rows * Hk / 192 >= 768)) return 3;
  return split || rows * Hk / 128 >= 384 ? 2 : 1;
}
constexpr AttnTuning kFp4Tuning = {1024, 256, 4, 384, fp4_tile_rows};

}  // namespace ssn
