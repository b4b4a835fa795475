// The paged attention's tile kernel for bf16 storage.
#include "attn_tiles.h"

namespace ssn {

hipError_t launch_attn_tiles_bf16(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const bool one = p.tiles.blocks == 1;
  if (a.D <= 64) return one ? launch_tiles<uint16_t, 64, 1>(a, p, st) : launch_tiles<uint16_t, 64, 2>(a, p, st);
  if (a.D <= 128) return one ? launch_tiles<uint16_t, 128, 1>(a, p, st) : launch_tiles<uint16_t, 128, 2>(a, p, st);
  return launch_tiles<uint16_t, 256, 1>(a, p, st);
}

}  // namespace ssn
