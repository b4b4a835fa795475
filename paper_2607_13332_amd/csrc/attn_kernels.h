// The paged attention's kernels: tiles, rows, or both in one launch.
#pragma once

#include "attn_plan.h"
#include "attn_rows.h"
#include "attn_tiles.h"

namespace ssn {

// Blocks of a compute unit: two where 256 registers hold a wave's rows (and, in
// the rows kernel, its keys and values: float32, 16 single tokens over up to 8192
// keys, 8 heads of 128: 128 us with two, 155 with one; bf16 rows of 32 or heads
// of 256 spill with two: 118 us became 190, 87 became 140, with probabilities in one part).
template <typename T, int DT, int QB>
constexpr int rows_blocks() { return DT * (int)sizeof(T) * QB <= (sizeof(T) == 4 ? 512 : 256) ? 2 : 1; }
template <typename T, int DT>
constexpr int tiles_blocks() { return DT * (int)sizeof(T) <= 512 ? 2 : 1; }

template <typename T, int DT, int QB, bool EXACT>
__global__ __launch_bounds__(256, (rows_blocks<T, DT, QB>())) void paged_attn_rows(AttnArgs a, AttnPart part,
                                                                                  int few) {
  __shared__ __align__(1024) char lds[rows_lds<T, DT, QB>()];
  rows_block<T, DT, QB, EXACT>(a, part, few, blockIdx.x, lds);
}

template <typename T, int DT, int QB, bool EXACT>
__global__ __launch_bounds__(256, (tiles_blocks<T, DT>())) void paged_attn_tiles(AttnArgs a, AttnPart part,
                                                                                 int few, int slots) {
  __shared__ __align__(1024) char lds[tiles_lds<T, DT>()];
  TileCount count;
  count.count(a.pb, a.G, 64 * QB, few, slots);
  tiles_block<T, DT, QB, EXACT>(a, part, few, count, blockIdx.x, lds);
}

// Both in one launch: first the tiles' blocks, the longer ones (a chunk of 1000
// tokens and 15 single tokens over up to 4096 keys: 172 us, 199 with the two
// kinds in alternate rounds; either kind fills the chip's registers with two
// blocks to a compute unit, so one does not hide behind the other).
template <typename T, int DT>
constexpr int both_blocks() { return rows_blocks<T, DT, 1>() < tiles_blocks<T, DT>() ? rows_blocks<T, DT, 1>() : tiles_blocks<T, DT>(); }
template <typename T, int DT, int QB, bool EXACT>
__global__ __launch_bounds__(256, (both_blocks<T, DT>())) void paged_attn_both(AttnArgs a, AttnPlan p, int slots,
                                                                               int rows) {
  constexpr int kLds = tiles_lds<T, DT>() > rows_lds<T, DT, 1>() ? tiles_lds<T, DT>() : rows_lds<T, DT, 1>();
  __shared__ __align__(1024) char lds[kLds];
  TileCount count;
  count.count(a.pb, a.G, 64 * QB, p.few, slots);
  const int tiles = count.total * a.Hk * p.tiles.ranges, id = blockIdx.x;
  if (id < tiles) tiles_block<T, DT, QB, EXACT>(a, p.tiles, p.few, count, id, lds);
  else if (id - tiles < rows) rows_block<T, DT, 1, EXACT>(a, p.rows, p.few, id - tiles, lds);
}

template <typename T, int DT, int QB, bool EXACT>
static hipError_t launch_rows(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_rows<T, DT, QB, EXACT>), dim3((unsigned)row_blocks(p, a.pb.B, a.Hk)), dim3(256), 0,
                     st, a, p.rows, p.few);
  return hipGetLastError();
}
template <typename T, int DT, int QB, bool EXACT>
static hipError_t launch_tiles(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const int64_t slots = tile_slots(a.pb.N, a.pb.B, a.G, 64 * QB), tiles = tile_blocks(p, a.pb.N, a.pb.B, a.Hk, a.G);
  if (p.rows.blocks) {
    const int64_t rows = row_blocks(p, a.pb.B, a.Hk);
    hipLaunchKernelGGL((paged_attn_both<T, DT, QB, EXACT>), dim3((unsigned)(tiles + rows)), dim3(256), 0, st, a, p,
                       (int)slots, (int)rows);
  } else {
    hipLaunchKernelGGL((paged_attn_tiles<T, DT, QB, EXACT>), dim3((unsigned)tiles), dim3(256), 0, st, a, p.tiles,
                       p.few, (int)slots);
  }
  return hipGetLastError();
}
// For a.D == DT and for the heads padded to DT in registers and LDS.
#define SSN_ATTN_EXACT(launch, T, DT, QB) \
  (a.D == DT ? launch<T, DT, QB, true>(a, p, st) : launch<T, DT, QB, false>(a, p, st))

}  // namespace ssn
