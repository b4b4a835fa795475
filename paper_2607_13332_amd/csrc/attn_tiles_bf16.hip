// The paged attention's tile kernel (and with it the rows kernel, where a batch
// has both) for bf16 storage.
#include "attn_kernels.h"

namespace ssn {

hipError_t launch_attn_tiles_bf16(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  if (a.D <= 64)
    return p.tiles.blocks == 1 ? SSN_ATTN_EXACT(launch_tiles, uint16_t, 64, 1)
                               : SSN_ATTN_EXACT(launch_tiles, uint16_t, 64, 2);
  if (a.D <= 128)
    return p.tiles.blocks == 1 ? SSN_ATTN_EXACT(launch_tiles, uint16_t, 128, 1)
         : p.tiles.blocks == 2 ? SSN_ATTN_EXACT(launch_tiles, uint16_t, 128, 2)
                               : SSN_ATTN_EXACT(launch_tiles, uint16_t, 128, 3);
  return SSN_ATTN_EXACT(launch_tiles, uint16_t, 256, 1);
}

}  // namespace ssn
