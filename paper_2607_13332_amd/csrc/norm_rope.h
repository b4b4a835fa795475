// Norms of heads with the position rotation: the pieces that the kernels of
// rows, of their gradients and of cache appends share.
#pragma once

#include <initializer_list>

#include "attn_device.h"
#include "ssn_launch.h"

namespace ssn {

// Of the generic kernels: a wave owns one head, lane l its elements l, l + 64, ...
constexpr int kGenericElems = 16;     // per lane: D <= 1024

struct RotPair {
  int other;        // the partner's element, or the element itself past R
  float c, s;       // y = x c + other s
};
// sign +1: rotation, -1: its transpose
__device__ __forceinline__ RotPair rot_pair(const NormRope& nr, const float* __restrict__ row, int e,
                                            float sign) {
  if (e >= nr.R) return RotPair{e, 1.f, 0.f};
  const int half = nr.R / 2;
  const int i = nr.pairs ? e >> 1 : (e < half ? e : e - half);
  const bool first = nr.pairs ? !(e & 1) : e < half;
  const int other = nr.pairs ? e ^ 1 : (first ? e + half : e - half);
  const float s = row[half + i] * sign;
  return RotPair{other, row[i], first ? -s : s};
}

template <typename T>
__device__ __forceinline__ float head_rms_inv(const T* __restrict__ x, int D, float eps, int lane) {
  if (eps < 0.f) return 1.f;
  float ss = 0.f;
  for (int e = lane; e < D; e += kWave) {
    const float v = load_as_f32(x + e);
    ss += v * v;
  }
  return 1.f / sqrtf(wave_sum(ss) / (float)D + eps);
}

template <typename T>
__device__ __forceinline__ float weight_at(const T* __restrict__ w, int e) {
  return w ? load_as_f32(w + e) : 1.f;
}

// put(e, value) for the elements of a normed and rotated head that the lane has.
template <typename T, typename F>
__device__ __forceinline__ void norm_rope_each(const NormRope& nr, const T* __restrict__ x,
                                               const T* __restrict__ w, const float* __restrict__ row, int lane,
                                               F put) {
  const float r = head_rms_inv(x, nr.D, nr.eps, lane);
  for (int e = lane; e < nr.D; e += kWave) {
    const RotPair rp = rot_pair(nr, row, e, 1.f);
    float v = load_as_f32(x + e) * r * weight_at(w, e) * rp.c;
    if (rp.other != e) v += load_as_f32(x + rp.other) * r * weight_at(w, rp.other) * rp.s;
    put(e, v);
  }
}
template <typename T>
__device__ __forceinline__ void norm_rope_head(const NormRope& nr, const T* __restrict__ x,
                                               const T* __restrict__ w, const float* __restrict__ row,
                                               T* __restrict__ y, int lane) {
  norm_rope_each(nr, x, w, row, lane, [&](int e, float v) { store_from_f32(y + e, v); });
}

template <typename T>
__device__ __forceinline__ const T* head_ptr(const HeadRows& r, int64_t i, int h, int D) {
  return (const T*)r.p + i * r.ld + (int64_t)h * D;
}

// Of the fast kernels: a lane's two 16-byte chunks of a head.
template <typename T>
struct Chunk {
  static constexpr int E = 16 / (int)sizeof(T);
  float v[E];
  __device__ __forceinline__ void set(u32x4 w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (E == 8) {
        v[2 * i] = lo_bf16(w[i]);
        v[2 * i + 1] = hi_bf16(w[i]);
      } else {
        v[i] = __uint_as_float(w[i]);
      }
    }
  }
  __device__ __forceinline__ u32x4 get() const {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (E == 8) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
      else w[i] = __float_as_uint(v[i]);
    }
    return w;
  }
  __device__ __forceinline__ void ones() {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = 1.f;
  }
};

enum { kNoRotation, kHalves, kPairs };

// Cosines and sines of a lane's pairs: E of each (halves: of the pairs of the
// two chunks; pairs: E / 2 of the first chunk, then E / 2 of the second).
template <typename T, int D, int ROT>
struct Turn {
  static constexpr int E = Chunk<T>::E;
  float c[E], s[E];
  __device__ __forceinline__ void load(const float* __restrict__ row, int j) {
    if constexpr (ROT == kHalves) {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        *(f32x4*)(c + e) = *(const f32x4*)(row + E * j + e);
        *(f32x4*)(s + e) = *(const f32x4*)(row + D / 2 + E * j + e);
      }
    } else if constexpr (ROT == kPairs) {
      typedef float part __attribute__((ext_vector_type(E / 2)));
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        *(part*)(c + z * E / 2) = *(const part*)(row + z * D / 4 + E / 2 * j);
        *(part*)(s + z * E / 2) = *(const part*)(row + D / 2 + z * D / 4 + E / 2 * j);
      }
    }
  }
  // (sign -1: back)
  __device__ __forceinline__ void apply(Chunk<T>& a, Chunk<T>& b, float sign) const {
    if constexpr (ROT == kHalves) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = a.v[e], y = b.v[e], t = s[e] * sign;
        a.v[e] = x * c[e] - y * t;
        b.v[e] = y * c[e] + x * t;
      }
    } else if constexpr (ROT == kPairs) {
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          Chunk<T>& h = z ? b : a;
          const float x = h.v[2 * e], y = h.v[2 * e + 1], t = s[z * E / 2 + e] * sign, u = c[z * E / 2 + e];
          h.v[2 * e] = x * u - y * t;
          h.v[2 * e + 1] = y * u + x * t;
        }
      }
    }
  }
};

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int m = LPH / 2; m >= 1; m >>= 1) v += __shfl_xor(v, m, kWave);
  return v;
}

// Waves of a launch: `passes` for each of `slots` tokens; a wave goes on to
// token + slots.  A wave does not change its pass: a launch has waves() of them.
struct Spread {
  int passes, slots;
  __host__ __device__ int64_t waves() const { return (int64_t)passes * slots; }
};
// (max_waves for the forward: appends of 11425 tokens take 88 / 82 / 72 / 69 / 76
// us for 4096 / 8192 / 16384 / 32768 / 131072 waves; the norms alone do not mind)
constexpr int64_t kForwardWaves = 32768;
inline Spread spread_tokens(int64_t N, int heads, int heads_per_wave, int64_t max_waves) {
  Spread s;
  s.passes = (heads + heads_per_wave - 1) / heads_per_wave;
  const int64_t most = max_waves / s.passes > 1 ? max_waves / s.passes : 1;
  s.slots = (int)(N < most ? N : most);
  return s;
}

inline bool aligned16(const HeadRows& r, int64_t s) {
  return r.H == 0 || ((uintptr_t)r.p % 16 == 0 && (r.ld * s) % 16 == 0);
}
inline bool fast_heads(int dtype, const NormRope& nr, std::initializer_list<HeadRows> rows,
                       std::initializer_list<const void*> ptrs) {
  if ((nr.D != 64 && nr.D != 128 && nr.D != 256) || (nr.R != 0 && nr.R != nr.D)) return false;
  for (const HeadRows& r : rows)
    if (!aligned16(r, dtype == kBF16 ? 2 : 4)) return false;
  for (const void* p : ptrs)
    if ((uintptr_t)p % 16) return false;
  return (uintptr_t)nr.table % 16 == 0;
}

inline unsigned wave_blocks(int64_t waves) {
  const int64_t b = (waves + 3) / 4;
  return (unsigned)(b < 1 ? 1 : (b > (1 << 20) ? (1 << 20) : b));
}

}  // namespace ssn
