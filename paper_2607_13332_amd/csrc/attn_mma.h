// Matrix-core pieces shared by the paged attention kernels.
//
// Both products are taken transposed, with 16 x 16 tiles:
//   S^T (keys x rows)  = K Q^T      A = K,   B = Q^T
//   O^T (d x rows)    += V^T P^T    A = V^T, B = P^T
// A lane holds one row (a query of one head: column lane % 16) in every
// accumulator: of S^T the keys 4 (lane / 16) + i of a tile, so that a row's
// maximum and sum are taken in registers and over the four lanes of a column
// only, and its probabilities are the B operand of the second product as they
// stand -- a K slot's key is free to choose as long as V^T carries the same.
//
// An operand fragment is 16 bytes a lane for either type.  bf16: 8 values, one
// 16x16x32 instruction.  float32: 4 values, four 16x16x4 instructions, the
// i-th with element i of every lane.
#pragma once

#include "attn_device.h"

namespace ssn {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegInf = -__builtin_inff();

// A cache row in LDS is RB bytes in 16-byte chunks, chunk c of key k at
// position c ^ swizzle(k).  LDS serves 8 lanes' 16 bytes or 16 lanes' 8 bytes a
// cycle, 128 bytes: of K's rows the equal chunks of 8 consecutive keys have to
// fall into different columns of 16 bytes, of V's the 32-byte pieces of 4
// consecutive keys.  Conflicts counted by rocprofv3, of the LDS cycles: none in
// bf16 (30 % with V's order for both), 38 % in float32, whose LDS cycles are 15 %
// of the kernel's.
template <int RB>
__device__ __forceinline__ uint32_t swizzle_keys(uint32_t k) {
  return RB >= 256 ? k & 15 : k & 7;
}
template <int RB>
__device__ __forceinline__ uint32_t swizzle_values(uint32_t k) {
  if constexpr (RB >= 256) return ((k & 7) << 1) | ((k >> 3) & 1);
  else return (((k >> 1) & 3) << 1) | ((k >> 3) & 1);
}

template <typename T>
struct Mma;

template <>
struct Mma<uint16_t> {
  static constexpr int kKeys = 32;         // keys of one step of the second product
  __device__ static __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) { return mfma16x16x32(a, b, c); }
  // Probabilities of a step from its tiles of S^T, rounded to bf16 (nearest
  // even): off by 2^-8 of each at most, as the rounded output is.
  __device__ static __forceinline__ u32x4 probs(const f32x4* s) {
    return u32x4{pack_bf16x2(s[0][0], s[0][1]), pack_bf16x2(s[0][2], s[0][3]), pack_bf16x2(s[1][0], s[1][1]),
                 pack_bf16x2(s[1][2], s[1][3])};
  }
  // What that rounding left, rounded in turn: with both a probability is off by
  // 2^-16 at most, and its product with V is a float32 one for all that shows.
  __device__ static __forceinline__ u32x4 remainders(const f32x4* s, u32x4 p) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = pack_bf16x2(s[i >> 1][2 * (i & 1)] - lo_bf16(p[i]), s[i >> 1][2 * (i & 1) + 1] - hi_bf16(p[i]));
    return r;
  }
  static constexpr int kParts = 2;         // of a probability, where a kernel takes them
  static constexpr int kTiles = 2;         // tiles of S^T in a step
  // V^T of 16 d's for a step: lane's d = 16 dt + lane % 16, its keys 4 (lane /
  // 16) + i of the step's two tiles.  `vb`: vbase() of the lane.
  template <int RB>
  __device__ static __forceinline__ uint32_t vbase(int lane, int) {
    const int L = lane & 15, key = 4 * (lane >> 4) + (L >> 2);
    return key * RB + ((((uint32_t)(L & 3) >> 1) ^ swizzle_values<RB>(key)) << 4) + (L & 1) * 8;
  }
  static constexpr int kBases = 1;
  template <int RB>
  __device__ static __forceinline__ u32x4 vfrag(const char* lds, const uint32_t* vb, int step, int dt) {
    const char* p = lds + (vb[0] ^ (uint32_t)(dt * 32)) + step * 32 * RB;
    const u32x2 a = lds_read_tr16((const uint16_t*)p), b = lds_read_tr16((const uint16_t*)(p + 16 * RB));
    return u32x4{a[0], a[1], b[0], b[1]};
  }
  // v with infinities and NaN as the largest numbers of their sign: as unsigned
  // numbers they are the largest of the negative ones, as signed of the others.
  __device__ static __forceinline__ u32x4 bounded(u32x4 v) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = v[i];         // (a bit cast of the element itself takes the first one)
      const u16x2 n = __builtin_elementwise_min(__builtin_bit_cast(u16x2, w), u16x2{0xFF7F, 0xFF7F});
      v[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, n), i16x2{0x7F7F, 0x7F7F}));
    }
    return v;
  }
  // v with infinities and NaN as zeros.
  __device__ static __forceinline__ u32x4 finite_part(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = (v[i] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu;
      const uint32_t hi = (v[i] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u;
      v[i] &= lo | hi;
    }
    return v;
  }
};

template <>
struct Mma<float> {
  static constexpr int kKeys = 16;
  __device__ static __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mfma16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c);
    return c;
  }
  __device__ static __forceinline__ u32x4 probs(const f32x4* s) { return __builtin_bit_cast(u32x4, s[0]); }
  static constexpr int kParts = 1;
  static constexpr int kTiles = 1;
  template <int RB>
  __device__ static __forceinline__ uint32_t vbase(int lane, int i) {
    const int L = lane & 15, key = 4 * (lane >> 4) + i;
    return key * RB + (((uint32_t)(L >> 2) ^ swizzle_values<RB>(key)) << 4) + (L & 3) * 4;
  }
  static constexpr int kBases = 4;
  template <int RB>
  __device__ static __forceinline__ u32x4 vfrag(const char* lds, const uint32_t* vb, int step, int dt) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = *(const uint32_t*)(lds + (vb[i] ^ (uint32_t)(dt * 64)) + step * 16 * RB);
    return v;
  }
  __device__ static __forceinline__ u32x4 finite_part(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (v[i] & 0x7F800000u) == 0x7F800000u ? 0u : v[i];
    return v;
  }
};

// What a wave keeps of 16 QB rows: m (the score the sums are taken
// against, before the scale; the same in the four lanes of a column), l (this
// lane's share of the sum of exp2((s - m) c)) and O^T.
template <int DT16, int QB>
struct RowState {
  f32x4 o[DT16][QB];
  float m[QB], l[QB];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      m[q] = kNegInf;
      l[q] = 0.f;
#pragma unroll
      for (int d = 0; d < DT16; ++d) o[d][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// Scores to probabilities exp2((s - m) c), as the B operands of the second
// product, and l += their sum.  m does not follow the maximum: the sums are the
// same against any m, so a row's moves (and its l and O are rescaled) only where
// it has not been set, or where a lane's sum of probabilities passes kFar; no
// maximum is taken otherwise.  Rows do not touch each other's bits.
constexpr float kFar = 1024.f;
__device__ __forceinline__ bool far(float sum, float m) { return !(sum <= kFar) || m == kNegInf; }
// PARTS of a probability: it as it is rounded, then what the rounding left.
template <typename T, int PARTS, int NKB, int QB>
__device__ __forceinline__ bool probabilities(const f32x4 (&s)[NKB][QB], const float (&m)[QB], float c,
                                              u32x4 (&p)[PARTS][NKB / Mma<T>::kTiles][QB], float (&sum)[QB]) {
  using M = Mma<T>;
  bool any = false;
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    // nothing seen so far: exp2 of -inf - 0 is 0
    const float base = (m[q] == kNegInf ? 0.f : m[q]) * c;
    sum[q] = 0.f;
#pragma unroll
    for (int t = 0; t < NKB / M::kTiles; ++t) {
      f32x4 x[M::kTiles];
#pragma unroll
      for (int u = 0; u < M::kTiles; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t * M::kTiles + u][q][i], c, -base));
          sum[q] += x[u][i];
        }
      p[0][t][q] = M::probs(x);
      if constexpr (PARTS == 2) p[1][t][q] = M::remainders(x, p[0][t][q]);
    }
    any |= far(sum[q], m[q]);
  }
  return any;
}
template <typename T, int PARTS, int NKB, int DT16, int QB>
__device__ __forceinline__ void softmax_step(const f32x4 (&s)[NKB][QB], RowState<DT16, QB>& st, float c,
                                             u32x4 (&p)[PARTS][NKB / Mma<T>::kTiles][QB]) {
  float sum[QB];
  if (__any(probabilities<T, PARTS>(s, st.m, c, p, sum))) {
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      int move = far(sum[q], st.m[q]);
      move |= __shfl_xor(move, 16, kWave);
      move |= __shfl_xor(move, 32, kWave);
      float m = s[0][q][0];
#pragma unroll
      for (int k = 0; k < NKB; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, s[k][q][i]);
      m = fmaxf(m, __shfl_xor(m, 16, kWave));
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      m = move ? fmaxf(m, st.m[q]) : st.m[q];
      const float fade = __builtin_amdgcn_exp2f((st.m[q] - (m == kNegInf ? 0.f : m)) * c);
      st.m[q] = m;
      st.l[q] *= fade;
#pragma unroll
      for (int d = 0; d < DT16; ++d) st.o[d][q] *= fade;
    }
    probabilities<T, PARTS>(s, st.m, c, p, sum);
  }
#pragma unroll
  for (int q = 0; q < QB; ++q) st.l[q] += sum[q];
}

// O^T += V^T P^T over NS steps of keys in LDS.  MASKED: some rows do not
// see some of its keys, and 0 times an infinity or a NaN there would reach
// them; what is not finite is left out (`odd` says so) for add_not_finite().
template <typename T, int RB, bool MASKED, int PARTS, int NS, int DT16, int QB>
__device__ __forceinline__ void weigh(const char* vlds, const uint32_t* vb, const u32x4 (&p)[PARTS][NS][QB],
                                      RowState<DT16, QB>& st, uint32_t& odd) {
  using M = Mma<T>;
#pragma unroll
  for (int t = 0; t < NS; ++t) {
#pragma unroll
    for (int d = 0; d < DT16; ++d) {
      u32x4 v = M::template vfrag<RB>(vlds, vb, t, d);
      if constexpr (MASKED) {
        const u32x4 f = M::finite_part(v);
        odd |= (f[0] ^ v[0]) | (f[1] ^ v[1]) | (f[2] ^ v[2]) | (f[3] ^ v[3]);
        v = f;
      }
      if constexpr (PARTS == 2) {
        // (a remainder may be zero or negative: an infinity times it would be NaN
        // or of the other sign)
        const u32x4 f = MASKED ? v : M::bounded(v);
#pragma unroll
        for (int q = 0; q < QB; ++q) st.o[d][q] = M::mma(f, p[1][t][q], st.o[d][q]);
      }
#pragma unroll
      for (int q = 0; q < QB; ++q) st.o[d][q] = M::mma(v, p[0][t][q], st.o[d][q]);
    }
  }
}

// The infinities and NaN that weigh<MASKED> left out of row `v` of V, for the
// rows of O that see it: their weight is positive, so each adds itself.
template <typename T, int DT16, int QB>
__device__ __forceinline__ void add_not_finite(const T* v, int D, const bool (&sees)[QB], RowState<DT16, QB>& st) {
  const int h4 = 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
  for (int d = 0; d < DT16; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 16 * d + h4 + i;
      const float x = e < D ? load_as_f32(v + e) : 0.f;
      const float y = fabsf(x) < __builtin_inff() ? 0.f : x;
#pragma unroll
      for (int q = 0; q < QB; ++q) st.o[d][q][i] += sees[q] ? y : 0.f;
    }
}

// The sum over the four lanes of a column.
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 2) *(u32x2*)p = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *(f32x4*)p = v;
}

}  // namespace ssn
