// Device-side helpers shared by the attention sublayer's kernels.
#pragma once

#include "attn_launch.h"
#include "ssn_device.h"

namespace ssn {

__device__ __forceinline__ uint32_t div_fast(const FastDiv& f, uint32_t x) {
  return (uint32_t)(((uint64_t)x * f.m) >> (31 + f.s));
}

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// One sequence of the batch: its rows [s0, s1) and its length, clamped so
// that every row and position they lead to exists.
struct Sequence {
  int s0, s1, len;
};
__device__ __forceinline__ Sequence sequence_of(const PagedBatch& pb, int b) {
  Sequence s;
  s.s0 = clampi(pb.starts[b], 0, pb.N);
  s.s1 = clampi(pb.starts[b + 1], s.s0, pb.N);
  s.len = clampi(pb.lens[b], 0, pb.max_len);
  return s;
}

// The last b in [0, B) with first(b) <= x, for ascending first(0) <= x: a whole
// wave looks, 64 candidates at a time (one round of loads for up to 64
// sequences).  Bounded for any contents.
template <typename F>
__device__ __forceinline__ int last_at_most(int B, int x, F first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lane * step;
    const int hits = __popcll(__ballot(at < n && first(lo + (at < n ? at : 0)) <= x));
    const int skip = (hits > 0 ? hits - 1 : 0) * step;
    lo += skip;
    n = n - skip < step ? n - skip : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The sequence that row i belongs to (its end is past i unless i is padding);
// -1 before the first.  For a whole wave.
__device__ __forceinline__ int sequence_of_row(const PagedBatch& pb, int i) {
  if (i < pb.starts[0]) return -1;
  return last_at_most(pb.B, i, [&](int b) { return pb.starts[b]; });
}

// Row of D elements of the cache (of npages * Hk * page_size such rows) that
// holds position t of sequence b, head h; t < width * page_size.  In two
// steps, so that the page number can be on its way while other work is done.
struct Slot {
  int32_t page;
  uint32_t off;
};
__device__ __forceinline__ Slot find_slot(const PagedBatch& pb, int b, int t) {
  const uint32_t j = div_fast(pb.page, (uint32_t)t);
  return Slot{pb.pages[(int64_t)b * pb.width + j], (uint32_t)t - j * pb.page.d};
}
__device__ __forceinline__ uint32_t slot_row(const PagedBatch& pb, const Slot& s, int Hk, int h) {
  return ((uint32_t)clampi(s.page, 0, pb.npages - 1) * (uint32_t)Hk + (uint32_t)h) * pb.page.d + s.off;
}
__device__ __forceinline__ uint32_t cache_row(const PagedBatch& pb, int b, int Hk, int h, int t) {
  return slot_row(pb, find_slot(pb, b, t), Hk, h);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, kWave));
  return v;
}

}  // namespace ssn
