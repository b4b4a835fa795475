// The kernels of attention over a 4-bit cache: tiles, rows, or both in one launch.
#pragma once

#include "attn_plan.h"
#include "fp4_attn_rows.h"
#include "fp4_attn_tiles.h"

namespace ssn {

// Blocks of a compute unit: what its LDS holds, three at most (64 single tokens over
// caches of 1 to 4096 keys, 8 heads of 128: the rows kernel as it was with queries in
// registers 49 us with two, 44 with three; with the registers of four it gains
// nothing).
constexpr int kUnitLds = 160 * 1024;
template <typename T, int DT, int QB>
constexpr int fp4_rows_blocks() {
  constexpr int n = kUnitLds / fp4_rows_lds<T, DT, QB>();
  return n < 3 ? n : 3;
}
template <typename T, int DT>
constexpr int fp4_tiles_blocks() { return DT <= 128 ? 2 : 1; }

template <typename T, int DT, int QB, bool EXACT>
__global__ __launch_bounds__(256, (fp4_rows_blocks<T, DT, QB>())) void paged_attn_fp4_rows(Fp4AttnArgs a,
                                                                                          AttnPart part, int few) {
  __shared__ __align__(1024) char lds[fp4_rows_lds<T, DT, QB>()];
  fp4_rows_block<T, DT, QB, EXACT>(a, part, few, blockIdx.x, lds);
}

template <typename T, int DT, int QB, bool EXACT>
__global__ __launch_bounds__(256, (fp4_tiles_blocks<T, DT>())) void paged_attn_fp4_tiles(Fp4AttnArgs a, AttnPart part,
                                                                                         int few, int slots) {
  __shared__ __align__(1024) char lds[fp4_tiles_lds<DT>()];
  TileCount count;
  count.count(a.a.pb, a.a.G, 64 * QB, few, slots);
  fp4_tiles_block<T, DT, QB, EXACT>(a, part, few, count, blockIdx.x, lds);
}

// Both in one launch, the tiles' blocks first.
template <typename T, int DT>
constexpr int fp4_both_blocks() { return fp4_rows_blocks<T, DT, 1>() < fp4_tiles_blocks<T, DT>() ? fp4_rows_blocks<T, DT, 1>() : fp4_tiles_blocks<T, DT>(); }
template <typename T, int DT, int QB, bool EXACT>
__global__ __launch_bounds__(256, (fp4_both_blocks<T, DT>())) void paged_attn_fp4_both(Fp4AttnArgs a, AttnPlan p,
                                                                                       int slots, int rows) {
  constexpr int kLds = fp4_tiles_lds<DT>() > fp4_rows_lds<T, DT, 1>() ? fp4_tiles_lds<DT>() : fp4_rows_lds<T, DT, 1>();
  __shared__ __align__(1024) char lds[kLds];
  TileCount count;
  count.count(a.a.pb, a.a.G, 64 * QB, p.few, slots);
  const int tiles = count.total * a.a.Hk * p.tiles.ranges, id = blockIdx.x;
  if (id < tiles) fp4_tiles_block<T, DT, QB, EXACT>(a, p.tiles, p.few, count, id, lds);
  else if (id - tiles < rows) fp4_rows_block<T, DT, 1, EXACT>(a, p.rows, p.few, id - tiles, lds);
}

template <typename T, int DT, int QB, bool EXACT>
static hipError_t launch_fp4_rows(const Fp4AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_fp4_rows<T, DT, QB, EXACT>), dim3((unsigned)row_blocks(p, a.a.pb.B, a.a.Hk)),
                     dim3(256), 0, st, a, p.rows, p.few);
  return hipGetLastError();
}
template <typename T, int DT, int QB, bool EXACT>
static hipError_t launch_fp4_tiles(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st) {
  const AttnArgs& a = f.a;
  const int64_t slots = tile_slots(a.pb.N, a.pb.B, a.G, 64 * QB), tiles = tile_blocks(p, a.pb.N, a.pb.B, a.Hk, a.G);
  if (p.rows.blocks) {
    const int64_t rows = row_blocks(p, a.pb.B, a.Hk);
    hipLaunchKernelGGL((paged_attn_fp4_both<T, DT, QB, EXACT>), dim3((unsigned)(tiles + rows)), dim3(256), 0, st, f, p,
                       (int)slots, (int)rows);
  } else {
    hipLaunchKernelGGL((paged_attn_fp4_tiles<T, DT, QB, EXACT>), dim3((unsigned)tiles), dim3(256), 0, st, f, p.tiles,
                       p.few, (int)slots);
  }
  return hipGetLastError();
}
// For a.D == DT and for the heads padded to DT in registers and LDS.
#define SSN_FP4_EXACT(launch, T, DT, QB) \
  (f.a.D == DT ? launch<T, DT, QB, true>(f, p, st) : launch<T, DT, QB, false>(f, p, st))

}  // namespace ssn
