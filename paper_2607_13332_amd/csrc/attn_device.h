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

// The sequence that row i belongs to: the last b with starts[b] <= i (its end
// is past i unless i is padding); -1 before the first.
__device__ __forceinline__ int sequence_of_row(const PagedBatch& pb, int i) {
  int lo = 0, hi = pb.B;           // starts[lo - 1] <= i < starts[hi]
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (pb.starts[mid] <= i) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

// Row of D elements of the cache (of npages * Hk * page_size such rows) that
// holds position t of sequence b, head h; t < width * page_size.
__device__ __forceinline__ uint32_t cache_row(const PagedBatch& pb, int b, int Hk, int h, int t) {
  const uint32_t j = div_fast(pb.page, (uint32_t)t);
  const int page = clampi(pb.pages[(int64_t)b * pb.width + j], 0, pb.npages - 1);
  return ((uint32_t)page * (uint32_t)Hk + (uint32_t)h) * pb.page.d + ((uint32_t)t - j * pb.page.d);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, kWave));
  return v;
}

}  // namespace ssn
