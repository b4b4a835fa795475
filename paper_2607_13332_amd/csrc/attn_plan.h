// How an attention call is run: which kernels, with what tiles, over which ranges
// of keys.  Host code only.
#pragma once

#include "attn_launch.h"
#include "ssn_launch.h"

namespace ssn {

constexpr int kMaxRanges = 256;
// A launch holds fewer than 2^32 threads, 2^24 blocks of 256.  The tiles get half
// of them; the rows' blocks are at most 2^22 + 2048 (the entry point keeps B Hk
// below 2^22, and ranges are for fewer than 2048 blocks).
constexpr int64_t kMaxTileBlocks = (int64_t)1 << 23;

// Numbers that the tiles of a launch may have: at least ceil(rows / BM) for every
// sequence.
inline int64_t tile_slots(int64_t N, int64_t B, int64_t G, int64_t BM) { return N * G / BM + B; }

// Bytes of a part's partial results.  The tiles' lie before the rows', and both
// are read 16 bytes at a time: a multiple of 16.
inline size_t stage_bytes(const AttnPart& p, int64_t D) {
  if (!p.blocks || p.ranges <= 1) return 0;
  return ((size_t)p.ranges * (size_t)p.stage_rows * (size_t)(D + 2) * 4 + 15) / 16 * 16;
}
// Ranges for about `want` of them, no more than `fit` bytes hold.  They divide
// max_len: under their own bound and under 131072, us, 512 tokens over 32768 keys
// take 366 and 964, 64 over 8192 36 and 130, 64 single tokens over caches of 1 to
// 4096 keys 108 and 129, one over 2011 keys 14 and 33.
inline void split_keys(AttnPart& p, int64_t want, int64_t unit, int64_t max_len, int64_t D, size_t fit) {
  const int64_t row_bytes = p.stage_rows * (D + 2) * 4;
  if (row_bytes > 0 && (size_t)want > fit / (size_t)row_bytes) want = (int64_t)(fit / (size_t)row_bytes);
  if (want > kMaxRanges) want = kMaxRanges;
  const int64_t len = max_len > 1 ? max_len : 1;
  int64_t chunk = want > 1 ? (len + want - 1) / want : len;
  chunk = (chunk + unit - 1) / unit * unit;
  p.chunk = (int)chunk;
  p.ranges = (int)((len + p.chunk - 1) / p.chunk);
}
// 16-row blocks of a tile kernel's wave, 1 to 3.  More rows make more of every
// key read from LDS, fewer make more blocks: tiles of 192 rows where they fill
// the chip one and a half times, of 128 where they fill three quarters of it
// (the two blocks of a compute unit counted), else of 64.  bf16, 40 / 8 heads of
// 128, one prompt, us for 64 / 128 / 192 rows: 1024 tokens 29 / 33 / 63, 2048
// 81 / 63 / 80, 4096 277 / 202 / 192.  Over long caches keys are split to fill
// the chip instead: 512 tokens over 32768 keys 583 / 356 / 314.  With heads of
// 64, 192 rows gain nothing; float32 takes 64 (2048 tokens of 16 heads of 64: 687
// us, 698 with 128 rows; 1024 tokens 80, 127).
// What the host knows of a batch's lengths is the caller's bound, and a loose one
// costs: one prompt of 1024 / 2048 / 4096 tokens takes 30 / 60 / 171 us under a bound
// of 4096 and 54 / 77 / 169 under 8192 or more (8 / 8 heads of 128: 28 / 40 / 79 and
// 42 / 70 / 137).
inline int tile_rows(int dtype, int64_t rows, int64_t most, int64_t Hk, int64_t D, int64_t max_len) {
  if (dtype != kBF16 || D > 128 || most <= 64) return 1;
  const bool split = max_len >= 8192;
  if (D > 64 && (split || rows * Hk / 192 >= 768)) return 3;
  return split || rows * Hk / 128 >= 384 ? 2 : 1;
}
// How a kernel's calls are cut: `blocks` of the rows kernel that ranges aim at, the keys
// of a range a multiple of `unit` and no fewer than `least` for each pair of a sequence
// and a key head (2048 suffice); `beside` blocks of the tile kernel where a launch has
// both; and its 16-row blocks of a wave.
struct AttnTuning {
  int64_t blocks, unit, least, beside;
  int (*tile_rows)(int dtype, int64_t rows, int64_t most, int64_t max_q, int64_t Hk, int64_t D, int64_t max_len);
};
inline int stored_tile_rows(int dtype, int64_t rows, int64_t most, int64_t, int64_t Hk, int64_t D, int64_t max_len) {
  return tile_rows(dtype, rows, most, Hk, D, max_len);
}
constexpr AttnTuning kStoredTuning = {2048, 128, 0, 512, stored_tile_rows};
inline AttnPlan attention_plan(int dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                               int64_t max_len, size_t ws_bytes, const AttnTuning& tuning = kStoredTuning) {
  AttnPlan p = {};
  ws_bytes = ws_bytes / 16 * 16;
  const int64_t G = Hq / Hk, most = max_q * G;
  const bool tiles = most > 32 || (most > 16 && D > 128);
  // the rows kernel takes all sequences, or the single tokens among longer
  // chunks (unless all have max_q)
  if (!tiles) p.few = most <= 16 ? 16 : 32;
  else if (G <= 16 && N != B * max_q) p.few = 16;
  p.rows.blocks = (p.few + 15) / 16;
  p.rows.stage_rows = B * Hk * 16 * p.rows.blocks;
  p.tiles.stage_rows = N * Hq;
  if (tiles) {
    const int64_t rows = (p.few && N - B >= 0 ? N - B + 1 : N) * G;
    p.tiles.blocks = tuning.tile_rows(dtype, rows, most, max_q, Hk, D, max_len);
    // two blocks to a compute unit, where the rows alone do not give them (512
    // tokens over 32768 keys: 497 us for 256 blocks, 317 for 512, 315 for 1024;
    // four chunks of up to 100 over 8192: 105, 76, 87)
    const int64_t blocks = (rows / (64 * p.tiles.blocks) + 1) * Hk;
    const int64_t full = p.rows.blocks ? tuning.beside : 512;
    int64_t want = blocks >= full ? 1 : full / blocks;
    // as many as the grid holds: it has a block for every range of every number a
    // tile may have, and sequences without new tokens have numbers too
    const int64_t most_ranges = kMaxTileBlocks / (tile_slots(N, B, G, 64 * p.tiles.blocks) * Hk);
    if (want > most_ranges) want = most_ranges > 1 ? most_ranges : 1;
    split_keys(p.tiles, want, 256, max_len, D, ws_bytes);
  }
  if (p.rows.blocks) {
    // about 2048 blocks, so that long and short caches spread evenly (64 caches of
    // 1 to 4096 keys: 125 / 116 / 105 / 107 / 120 us for 512 / 1024 / 2048 / 4096 /
    // 8192), and no more than 64 ranges to join where 512 blocks have them
    const size_t left = ws_bytes - stage_bytes(p.tiles, D);
    const int64_t pairs = B * Hk, full = 512 / pairs, want = (tuning.blocks + pairs - 1) / pairs;
    int64_t ranges = want > 64 && want > full ? (full > 64 ? full : 64) : want;
    const int64_t least = tuning.least * pairs < 2048 ? tuning.least * pairs : 2048;
    if (least && ranges > max_len / least) ranges = max_len / least > 1 ? max_len / least : 1;
    split_keys(p.rows, ranges, tuning.unit, max_len, D, left);
  }
  return p;
}

// Blocks of the two kernels' launches.
inline int64_t tile_blocks(const AttnPlan& p, int64_t N, int64_t B, int64_t Hk, int64_t G) {
  return p.tiles.blocks ? tile_slots(N, B, G, 64 * p.tiles.blocks) * Hk * p.tiles.ranges : 0;
}
inline int64_t row_blocks(const AttnPlan& p, int64_t B, int64_t Hk) {
  return p.rows.blocks ? B * Hk * p.rows.ranges : 0;
}

}  // namespace ssn
