// The 4-bit cache's tile kernel (and with it the rows kernel, where a batch has
// both) for queries and outputs in bf16.
#include "fp4_attn_kernels.h"

namespace ssn {

hipError_t launch_fp4_tiles_bf16(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st) {
  if (f.a.D <= 64)
    return p.tiles.blocks == 1 ? SSN_FP4_EXACT(launch_fp4_tiles, uint16_t, 64, 1)
                               : SSN_FP4_EXACT(launch_fp4_tiles, uint16_t, 64, 2);
  if (f.a.D <= 128)
    return p.tiles.blocks == 1 ? SSN_FP4_EXACT(launch_fp4_tiles, uint16_t, 128, 1)
         : p.tiles.blocks == 2 ? SSN_FP4_EXACT(launch_fp4_tiles, uint16_t, 128, 2)
                               : SSN_FP4_EXACT(launch_fp4_tiles, uint16_t, 128, 3);
  return SSN_FP4_EXACT(launch_fp4_tiles, uint16_t, 256, 1);
}

}  // namespace ssn
