// Matrix-core pieces of attention over a 4-bit cache.  Keys and values are exact
// in bf16, so both products run on the bf16 matrix instructions for either type of
// Q and O: float32 queries and probabilities go in three bf16 parts, which hold all
// their bits, against one of K and V.
#pragma once

#include "attn_mma.h"
#include "fp4.h"

namespace ssn {

// Storage T of queries and outputs over a 4-bit cache.
template <typename T>
struct OverFp4 {};
template <typename T>
struct Mma<OverFp4<T>> : Mma<uint16_t> {
  static constexpr int kQueries = sizeof(T) == 2 ? 1 : 3;     // bf16 parts of a query
  static constexpr int kRowsParts = sizeof(T) == 2 ? 2 : 3;   // of a probability: rows kernel, tile kernel
  static constexpr int kTilesParts = sizeof(T) == 2 ? 1 : 3;
  // what is left after two parts of a probability, exactly
  __device__ static __forceinline__ u32x4 last_remainders(const f32x4* s, u32x4 p, u32x4 r) {
    u32x4 l;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      l[i] = pack_bf16x2((s[i >> 1][2 * (i & 1)] - lo_bf16(p[i])) - lo_bf16(r[i]),
                         (s[i >> 1][2 * (i & 1) + 1] - hi_bf16(p[i])) - hi_bf16(r[i]));
    return l;
  }
  // (infinities, of scale bytes that appends do not write, may become NaN against a
  // second part that is zero or of the other sign: 64 single tokens take 48 us instead
  // of 44 with them bounded, four long ones 123 instead of 109)
  __device__ static __forceinline__ u32x4 bounded(u32x4 v) { return v; }
};

// Eight elements of a query, as they lie in memory (zeros unless `take`), and in
// bf16 parts.  Of float32 the first part is truncated, so that no finite number
// becomes infinite; below 2^-110 the last parts run out of bf16's range (an element is
// then off by 2^-134 at most).
template <typename T>
struct QueryChunk {
  u32x4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p, bool take) {
#pragma unroll
    for (int z = 0; z < (int)sizeof(T) / 2; ++z) v[z] = take ? *((const u32x4*)p + z) : u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void parts(uint32_t flip, u32x4 (&q)[Mma<OverFp4<T>>::kQueries]) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[0][i] = v[0][i] ^ flip;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t h[2];
        float r[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t w = v[i / 2][2 * (i % 2) + e] ^ flip, a = w & 0x7FFFFFFFu;
          h[e] = (w & 0xFFFF0000u) | (a > 0x7F800000u ? 0x400000u : 0u);
          r[e] = a >= 0x7F800000u ? 0.f : __uint_as_float(w) - __uint_as_float(h[e]);
        }
        const uint32_t m = pack_bf16x2(r[0], r[1]);
        q[0][i] = (h[0] >> 16) | h[1];
        q[1][i] = m;
        q[2][i] = pack_bf16x2(r[0] - lo_bf16(m), r[1] - hi_bf16(m));
      }
    }
  }
};

// What weigh<MASKED> left out of a row of V with these scales, for the rows of O that
// see it: groups of NaN, and those that may hold infinities count as such.
constexpr int kNotFinite = 253;        // from this scale byte on
template <int DT16, int QB>
__device__ __forceinline__ void add_not_finite_groups(const uint8_t* scales, int D, const bool (&sees)[QB],
                                               RowState<DT16, QB>& st) {
#pragma unroll
  for (int d = 0; d < DT16; ++d)
    if (16 * d < D && scales[d / 2] >= kNotFinite) {
#pragma unroll
      for (int q = 0; q < QB; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[d][q][i] += sees[q] ? __builtin_nanf("") : 0.f;
    }
}

// The row of LDS that holds key l of 16's values: rows of 8 consecutive keys take a
// chunk each to different columns (swizzle_values), and a transposing read, which is
// served 256 bytes at a time, finds the pieces of 8 consecutive keys in different ones
// too.  (With rows 0-3, 8-11, 4-7, 12-15 it does not: 25 % of the tile kernel's LDS
// cycles were conflicts.)
__device__ __forceinline__ int value_row(int l) { return l ^ ((l & 4) << 1); }
// Mma::vbase() with the keys in these rows.
template <int RB>
__device__ __forceinline__ uint32_t value_base(int lane) {
  const int L = lane & 15, row = value_row(4 * (lane >> 4) + (L >> 2));
  return row * RB + ((((uint32_t)(L & 3) >> 1) ^ swizzle_values<RB>(row)) << 4) + (L & 1) * 8;
}

}  // namespace ssn
