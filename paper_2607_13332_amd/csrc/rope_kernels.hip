// Norms of heads with the position rotation, forward and backward, and the
// serving form that writes keys and values into a paged cache.
//
// A head x of D values at position p, in float32:
//   r = (mean(x^2) + eps)^-1/2,  n = x r w,  y = rot_p(n)
// and for g = rot_p^T(dL/dy), h = g w:
//   dL/dx = r (h - x r mean(h x r)),   dL/dw = sum over rows of g x r
#include <initializer_list>

#include "attn_device.h"
#include "ssn_launch.h"

namespace ssn {

__global__ __launch_bounds__(256) void rope_table_kernel(float* __restrict__ table, int64_t P, int64_t half,
                                                         double log_theta) {
  const int64_t n = P * half;
  for (int64_t e = blockIdx.x * (int64_t)256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
    const int64_t p = e / half, i = e - p * half;
    double s, c;
    sincos((double)p * exp(-log_theta * (double)i / (double)half), &s, &c);
    table[p * 2 * half + i] = (float)c;
    table[p * 2 * half + half + i] = (float)s;
  }
}

hipError_t launch_rope_table(int64_t P, int64_t R, double theta, float* table, hipStream_t st) {
  const int64_t n = P * (R / 2), blocks = (n + 255) / 256;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)(blocks > 65536 ? 65536 : blocks)), dim3(256), 0, st,
                     table, P, R / 2, log(theta));
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Generic kernels (any D up to 1024, any R, any alignment): a wave owns one
// head, lane l its elements l, l + 64, ...  An element's rotation partner is
// read again from memory (the cache holds it).
// ---------------------------------------------------------------------------
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

template <typename T>
__device__ __forceinline__ void norm_rope_head(const NormRope& nr, const T* __restrict__ x,
                                               const T* __restrict__ w, const float* __restrict__ row,
                                               T* __restrict__ y, int lane) {
  const float r = head_rms_inv(x, nr.D, nr.eps, lane);
  for (int e = lane; e < nr.D; e += kWave) {
    const RotPair rp = rot_pair(nr, row, e, 1.f);
    float v = load_as_f32(x + e) * r * weight_at(w, e) * rp.c;
    if (rp.other != e) v += load_as_f32(x + rp.other) * r * weight_at(w, rp.other) * rp.s;
    store_from_f32(y + e, v);
  }
}

template <typename T>
__device__ __forceinline__ const T* head_ptr(const HeadRows& r, int64_t i, int h, int D) {
  return (const T*)r.p + i * r.ld + (int64_t)h * D;
}

template <typename T>
__global__ __launch_bounds__(256) void norm_rope_generic(int N, NormRope nr, HeadRows q, HeadRows k,
                                                         const T* wq, const T* wk, const int32_t* pos,
                                                         HeadRows qo, HeadRows ko) {
  const int lane = threadIdx.x & 63, heads = q.H + k.H;
  const int64_t total = (int64_t)N * heads;
  for (int64_t j = blockIdx.x * 4LL + (threadIdx.x >> 6); j < total; j += gridDim.x * 4LL) {
    const int64_t i = j / heads;
    const int h = (int)(j - i * heads);
    const float* row = nr.R ? nr.table + (int64_t)clampi(pos[i], 0, nr.P - 1) * nr.R : nullptr;
    if (h < q.H)
      norm_rope_head(nr, head_ptr<T>(q, i, h, nr.D), wq, row, (T*)head_ptr<T>(qo, i, h, nr.D), lane);
    else
      norm_rope_head(nr, head_ptr<T>(k, i, h - q.H, nr.D), wk, row,
                     (T*)head_ptr<T>(ko, i, h - q.H, nr.D), lane);
  }
}

// A wave's share of dL/dw stays in its registers over all its heads; blocks
// add their waves' shares in order and leave them in ws [block][2][D].
template <typename T>
__global__ __launch_bounds__(256) void norm_rope_backward_generic(int N, NormRope nr, HeadRows q, HeadRows k,
                                                                  const T* wq, const T* wk,
                                                                  const int32_t* pos, HeadRows gq,
                                                                  HeadRows gk, HeadRows gqi, HeadRows gki,
                                                                  float* __restrict__ ws) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = q.H + k.H, D = nr.D;
  const int64_t total = (int64_t)N * heads;
  float gw[2][kGenericElems] = {};
  for (int64_t j = blockIdx.x * 4LL + wave; j < total; j += gridDim.x * 4LL) {
    const int64_t i = j / heads;
    const int h = (int)(j - i * heads);
    const bool isq = h < q.H;
    const T* x = isq ? head_ptr<T>(q, i, h, D) : head_ptr<T>(k, i, h - q.H, D);
    const T* gy = isq ? head_ptr<T>(gq, i, h, D) : head_ptr<T>(gk, i, h - q.H, D);
    T* gx = (T*)(isq ? head_ptr<T>(gqi, i, h, D) : head_ptr<T>(gki, i, h - q.H, D));
    const T* w = isq ? wq : wk;
    const float* row = nr.R ? nr.table + (int64_t)clampi(pos[i], 0, nr.P - 1) * nr.R : nullptr;
    const float r = head_rms_inv(x, D, nr.eps, lane);
    float g[kGenericElems], dot = 0.f;
#pragma unroll
    for (int m = 0; m < kGenericElems; ++m) {
      const int e = lane + m * kWave;
      g[m] = 0.f;
      if (e < D) {
        const RotPair rp = rot_pair(nr, row, e, -1.f);
        float v = load_as_f32(gy + e) * rp.c;
        if (rp.other != e) v += load_as_f32(gy + rp.other) * rp.s;
        const float n = load_as_f32(x + e) * r;
        if (isq) gw[0][m] += v * n;
        else gw[1][m] += v * n;
        g[m] = v * weight_at(w, e);
        dot += g[m] * n;
      }
    }
    const float mean = nr.eps < 0.f ? 0.f : wave_sum(dot) / (float)D;
#pragma unroll
    for (int m = 0; m < kGenericElems; ++m) {
      const int e = lane + m * kWave;
      if (e < D)
        store_from_f32(gx + e, nr.eps < 0.f ? g[m] : r * (g[m] - load_as_f32(x + e) * r * mean));
    }
  }
  if (!ws) return;
  __shared__ float part[4][1024];
#pragma unroll
  for (int z = 0; z < 2; ++z) {
#pragma unroll
    for (int m = 0; m < kGenericElems; ++m)
      if (lane + m * kWave < D) part[wave][lane + m * kWave] = gw[z][m];
    __syncthreads();
    for (int e = threadIdx.x; e < D; e += 256)
      ws[((int64_t)blockIdx.x * 2 + z) * D + e] = (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
    __syncthreads();
  }
}

// dL/dw = the blocks' shares, in block order: a block owns 16 columns of one
// weight, its 16 groups of lanes every 16th row, joined in order.
__global__ __launch_bounds__(256) void weight_grad_sum(const float* __restrict__ ws, int blocks, int D,
                                                       float* __restrict__ gwq, float* __restrict__ gwk) {
  __shared__ float part[16][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4, e = blockIdx.x * 16 + c;
  float* out = blockIdx.y ? gwk : gwq;
  float s = 0.f;
  if (e < D)
#pragma unroll 8
    for (int b = g; b < blocks; b += 16) s += ws[((int64_t)b * 2 + blockIdx.y) * D + e];
  part[g][c] = s;
  __syncthreads();
  if (g == 0 && e < D && out) {
    float t = 0.f;
    for (int m = 0; m < 16; ++m) t += part[m][c];
    out[e] = t;
  }
}

// Rows of a serving batch: queries to Qout, keys and values to their slots.
template <typename T>
__global__ __launch_bounds__(256) void kv_append_generic(PagedBatch pb, NormRope nr, HeadRows q, HeadRows k,
                                                         HeadRows v, const T* wq, const T* wk, T* Kc, T* Vc,
                                                         HeadRows qo) {
  const int lane = threadIdx.x & 63, heads = q.H + 2 * k.H, D = nr.D;
  const int64_t total = (int64_t)pb.N * heads;
  for (int64_t j = blockIdx.x * 4LL + (threadIdx.x >> 6); j < total; j += gridDim.x * 4LL) {
    const int i = (int)(j / heads), h = (int)(j - (int64_t)i * heads);
    const int b = sequence_of_row(pb, i);
    if (b < 0) continue;
    const Sequence sq = sequence_of(pb, b);
    const int p = sq.len - (sq.s1 - i);
    if (i >= sq.s1 || p < 0) continue;
    const float* row = nr.R ? nr.table + (int64_t)clampi(p, 0, nr.P - 1) * nr.R : nullptr;
    if (h < q.H) {
      norm_rope_head(nr, head_ptr<T>(q, i, h, D), wq, row, (T*)head_ptr<T>(qo, i, h, D), lane);
    } else if (h < q.H + k.H) {
      norm_rope_head(nr, head_ptr<T>(k, i, h - q.H, D), wk, row,
                     Kc + (int64_t)cache_row(pb, b, k.H, h - q.H, p) * D, lane);
    } else {
      const T* x = head_ptr<T>(v, i, h - q.H - k.H, D);
      T* y = Vc + (int64_t)cache_row(pb, b, k.H, h - q.H - k.H, p) * D;
      for (int e = lane; e < D; e += kWave) y[e] = x[e];
    }
  }
}

// ---------------------------------------------------------------------------
// Fast kernels (D = 64, 128, 256; the whole head rotated or none of it; 16-byte
// alignment).  Memory bounds them: every row is read once and written once.
//
// A lane holds two 16-byte chunks of a head, E elements each: E j .. and D/2 +
// E j .., j its place among the LPH lanes of the head.  With SSN_ROPE_HALVES the
// two chunks are each other's partners, with SSN_ROPE_PAIRS each is its own, so
// the rotation never leaves a lane; a head's sums take log2(LPH) exchanges.
// A wave covers 64 / LPH consecutive heads of a token (a pass; queries, then
// keys, then values) and keeps to its pass from token to token: its weights and
// its share of their gradients stay in registers, and the waves of a block read
// the same rows of the rotation table.
// ---------------------------------------------------------------------------
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
static Spread spread_tokens(int64_t N, int heads, int heads_per_wave, int64_t max_waves) {
  Spread s;
  s.passes = (heads + heads_per_wave - 1) / heads_per_wave;
  const int64_t most = max_waves / s.passes > 1 ? max_waves / s.passes : 1;
  s.slots = (int)(N < most ? N : most);
  return s;
}

// 4096 tokens of 40 + 8 heads of 128, bf16: 20.5 us, 5.0 TB/s.
// APPEND: keys and values go to their slots of the cache, positions follow
// from the batch, and the heads of v come after those of k.  Four prompts of
// 11425 tokens in all: 69 us, 5.3 TB/s; one token 3.2 us.
template <typename T, int D, int ROT, bool APPEND>
__global__ __launch_bounds__(256) void norm_rope_rows(int N, Spread sp, NormRope nr, HeadRows q, HeadRows k,
                                                      HeadRows v, const T* __restrict__ wq,
                                                      const T* __restrict__ wk,
                                                      const int32_t* __restrict__ pos, HeadRows qo,
                                                      HeadRows ko, PagedBatch pb, T* __restrict__ Kc,
                                                      T* __restrict__ Vc) {
  constexpr int E = Chunk<T>::E, LPH = D / (2 * E);
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (id >= sp.waves()) return;
  const int pass = id % sp.passes, j = lane % LPH, head = pass * (kWave / LPH) + lane / LPH;
  const bool isq = head < q.H, isk = !isq && head < q.H + k.H;
  const bool isv = APPEND && !isq && !isk && head < q.H + 2 * k.H, any = isq || isk || isv;
  const HeadRows in = isq ? q : (isv ? v : k);
  const int h = isq ? head : (isv ? head - q.H - k.H : head - q.H);
  const T* src = (const T*)in.p + h * D + E * j;
  Chunk<T> wa, wb;
  wa.ones();
  wb.ones();
  const T* w = isq ? wq : wk;
  if (any && !isv && w) {
    wa.set(*(const u32x4*)(w + E * j));
    wb.set(*(const u32x4*)(w + D / 2 + E * j));
  }
  for (int i = id / sp.passes; i < N; i += sp.slots) {
    int p = 0, b = 0;
    if constexpr (APPEND) {
      b = sequence_of_row(pb, i);
      if (b < 0) continue;
      const Sequence sq = sequence_of(pb, b);
      p = sq.len - (sq.s1 - i);
      if (i >= sq.s1 || p < 0) continue;
    } else if constexpr (ROT != kNoRotation) {
      p = pos[i];
    }
    u32x4 xa = {0, 0, 0, 0}, xb = {0, 0, 0, 0};
    if (any) {
      xa = __builtin_nontemporal_load((const u32x4*)(src + i * in.ld));
      xb = __builtin_nontemporal_load((const u32x4*)(src + i * in.ld + D / 2));
    }
    Turn<T, D, ROT> turn;
    if constexpr (ROT != kNoRotation) turn.load(nr.table + (int64_t)clampi(p, 0, nr.P - 1) * D, j);
    T* dst;
    if (isq) dst = (T*)qo.p + i * qo.ld + h * D;
    else if constexpr (APPEND) dst = (isv ? Vc : Kc) + (int64_t)cache_row(pb, b, k.H, any ? h : 0, p) * D;
    else dst = (T*)ko.p + i * ko.ld + h * D;
    if (!isv) {
      Chunk<T> a, c;
      a.set(xa);
      c.set(xb);
      if (nr.eps >= 0.f) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss += a.v[e] * a.v[e] + c.v[e] * c.v[e];
        const float r = rsqrtf(head_sum<LPH>(ss) * (1.f / D) + nr.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          a.v[e] *= r * wa.v[e];
          c.v[e] *= r * wb.v[e];
        }
      }
      turn.apply(a, c, 1.f);
      xa = a.get();
      xb = c.get();
    }
    if (any) {
      *(u32x4*)(dst + E * j) = xa;
      *(u32x4*)(dst + D / 2 + E * j) = xb;
    }
  }
}

// 12205 tokens of 40 + 8 heads of 128, bf16: 76 us, 5.9 TB/s, and 4.8 us for the
// sum of the blocks' shares of dL/dw.
constexpr int kBackWaves = 8;         // of a block
template <typename T, int D, int ROT>
__global__ __launch_bounds__(64 * kBackWaves) void norm_rope_backward_rows(
    int N, Spread sp, NormRope nr, HeadRows q, HeadRows k, const T* __restrict__ wq, const T* __restrict__ wk,
    const int32_t* __restrict__ pos, HeadRows gq, HeadRows gk, HeadRows gqi, HeadRows gki,
    float* __restrict__ ws) {
  constexpr int E = Chunk<T>::E, LPH = D / (2 * E);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int id = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kBackWaves + wave));
  const int pass = id % sp.passes, j = lane % LPH, head = pass * (kWave / LPH) + lane / LPH;
  const bool isq = head < q.H, any = head < q.H + k.H;
  const int h = isq ? head : head - q.H;
  const HeadRows in = isq ? q : k, gin = isq ? gq : gk, out = isq ? gqi : gki;
  const T* src = (const T*)in.p + h * D + E * j;
  const T* gsrc = (const T*)gin.p + h * D + E * j;
  T* dst = (T*)out.p + h * D + E * j;
  Chunk<T> wa, wb, ga, gb;              // ga, gb: shares of dL/dw
  wa.ones();
  wb.ones();
  const T* w = isq ? wq : wk;
  if (any && w) {
    wa.set(*(const u32x4*)(w + E * j));
    wb.set(*(const u32x4*)(w + D / 2 + E * j));
  }
#pragma unroll
  for (int e = 0; e < E; ++e) ga.v[e] = gb.v[e] = 0.f;
  const int first = id < sp.waves() ? id / sp.passes : N;
  for (int i = first; i < N; i += sp.slots) {
    u32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}}, y[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (any) {
      x[0] = __builtin_nontemporal_load((const u32x4*)(src + i * in.ld));
      x[1] = __builtin_nontemporal_load((const u32x4*)(src + i * in.ld + D / 2));
      y[0] = __builtin_nontemporal_load((const u32x4*)(gsrc + i * gin.ld));
      y[1] = __builtin_nontemporal_load((const u32x4*)(gsrc + i * gin.ld + D / 2));
    }
    Turn<T, D, ROT> turn;
    if constexpr (ROT != kNoRotation) turn.load(nr.table + (int64_t)clampi(pos[i], 0, nr.P - 1) * D, j);
    Chunk<T> xa, xb, a, b;
    xa.set(x[0]);
    xb.set(x[1]);
    a.set(y[0]);
    b.set(y[1]);
    turn.apply(a, b, -1.f);
    if (nr.eps >= 0.f) {
      float ss = 0.f, dot = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        ss += xa.v[e] * xa.v[e] + xb.v[e] * xb.v[e];
        dot += a.v[e] * wa.v[e] * xa.v[e] + b.v[e] * wb.v[e] * xb.v[e];
      }
      // (a lane without a head holds zeros: at eps = 0 their inverse root would be
      // infinite, and its products NaN in the shares of dL/dw)
      const float inv = rsqrtf(head_sum<LPH>(ss) * (1.f / D) + nr.eps), r = any ? inv : 0.f;
      // mean(h x r) r; r^3 by itself could leave float32 (heads of 1e-18, no eps)
      const float m = head_sum<LPH>(dot) * r * (1.f / D) * r;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float na = xa.v[e] * r, nb = xb.v[e] * r;
        ga.v[e] += a.v[e] * na;
        gb.v[e] += b.v[e] * nb;
        a.v[e] = a.v[e] * wa.v[e] * r - na * m;
        b.v[e] = b.v[e] * wb.v[e] * r - nb * m;
      }
    }
    if (any) {
      *(u32x4*)(dst + i * out.ld) = a.get();
      *(u32x4*)(dst + i * out.ld + D / 2) = b.get();
    }
  }
  if (!ws) return;
  // the heads of a wave, then the waves of a block in order
  __shared__ float part[kBackWaves][2][D];
#pragma unroll
  for (int z = 0; z < 2; ++z)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float s = (isq == (z == 0)) ? ga.v[e] : 0.f, t = (isq == (z == 0)) ? gb.v[e] : 0.f;
#pragma unroll
      for (int m = LPH; m < kWave; m <<= 1) {
        s += __shfl_xor(s, m, kWave);
        t += __shfl_xor(t, m, kWave);
      }
      if (lane < LPH) {
        part[wave][z][E * j + e] = s;
        part[wave][z][D / 2 + E * j + e] = t;
      }
    }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * D; e += 64 * kBackWaves) {
    float s = 0.f;
#pragma unroll
    for (int m = 0; m < kBackWaves; ++m) s += part[m][e / D][e % D];
    ws[(int64_t)blockIdx.x * 2 * D + e] = s;
  }
}

static bool aligned16(const HeadRows& r, int64_t s) {
  return r.H == 0 || ((uintptr_t)r.p % 16 == 0 && (r.ld * s) % 16 == 0);
}
static bool fast_heads(int dtype, const NormRope& nr, std::initializer_list<HeadRows> rows,
                       std::initializer_list<const void*> ptrs) {
  if ((nr.D != 64 && nr.D != 128 && nr.D != 256) || (nr.R != 0 && nr.R != nr.D)) return false;
  for (const HeadRows& r : rows)
    if (!aligned16(r, dtype == kBF16 ? 2 : 4)) return false;
  for (const void* p : ptrs)
    if ((uintptr_t)p % 16) return false;
  return (uintptr_t)nr.table % 16 == 0;
}

struct RowsLaunch {
  int64_t N;
  NormRope nr;
  HeadRows q, k, v;
  const void *wq, *wk;
  const int32_t* pos;
  HeadRows qo, ko;
  PagedBatch pb;
  void *Kc, *Vc;
  bool append;
  hipStream_t st;
};
template <typename T, int D, int ROT, bool APPEND>
static hipError_t launch_rows_kernel(const RowsLaunch& a) {
  const Spread sp = spread_tokens(a.N, a.q.H + (APPEND ? 2 : 1) * a.k.H, kWave * 2 * Chunk<T>::E / D,
                                  kForwardWaves);
  hipLaunchKernelGGL((norm_rope_rows<T, D, ROT, APPEND>), dim3((unsigned)((sp.waves() + 3) / 4)), dim3(256), 0,
                     a.st, (int)a.N, sp, a.nr, a.q, a.k, a.v, (const T*)a.wq, (const T*)a.wk, a.pos, a.qo, a.ko,
                     a.pb, (T*)a.Kc, (T*)a.Vc);
  return hipGetLastError();
}
template <typename T, int D, int ROT>
static hipError_t launch_rows_append(const RowsLaunch& a) {
  return a.append ? launch_rows_kernel<T, D, ROT, true>(a) : launch_rows_kernel<T, D, ROT, false>(a);
}
template <typename T, int D>
static hipError_t launch_rows_rot(const RowsLaunch& a) {
  if (!a.nr.R) return launch_rows_append<T, D, kNoRotation>(a);
  return a.nr.pairs ? launch_rows_append<T, D, kPairs>(a) : launch_rows_append<T, D, kHalves>(a);
}
template <typename T>
static hipError_t launch_rows_fast(const RowsLaunch& a) {
  if (a.nr.D == 64) return launch_rows_rot<T, 64>(a);
  return a.nr.D == 128 ? launch_rows_rot<T, 128>(a) : launch_rows_rot<T, 256>(a);
}

struct BackLaunch {
  int64_t N;
  NormRope nr;
  HeadRows q, k;
  const void *wq, *wk;
  const int32_t* pos;
  HeadRows gq, gk, gqi, gki;
  float* ws;
  int blocks;
  hipStream_t st;
};
template <typename T, int D, int ROT>
static hipError_t launch_back_kernel(const BackLaunch& a) {
  const Spread sp = spread_tokens(a.N, a.q.H + a.k.H, kWave * 2 * Chunk<T>::E / D, (int64_t)a.blocks * kBackWaves);
  hipLaunchKernelGGL((norm_rope_backward_rows<T, D, ROT>), dim3(a.blocks), dim3(64 * kBackWaves), 0, a.st,
                     (int)a.N, sp, a.nr, a.q, a.k, (const T*)a.wq, (const T*)a.wk, a.pos, a.gq, a.gk, a.gqi, a.gki,
                     a.ws);
  return hipGetLastError();
}
template <typename T, int D>
static hipError_t launch_back_rot(const BackLaunch& a) {
  if (!a.nr.R) return launch_back_kernel<T, D, kNoRotation>(a);
  return a.nr.pairs ? launch_back_kernel<T, D, kPairs>(a) : launch_back_kernel<T, D, kHalves>(a);
}
template <typename T>
static hipError_t launch_back_fast(const BackLaunch& a) {
  if (a.nr.D == 64) return launch_back_rot<T, 64>(a);
  return a.nr.D == 128 ? launch_back_rot<T, 128>(a) : launch_back_rot<T, 256>(a);
}

static unsigned wave_blocks(int64_t waves) {
  const int64_t b = (waves + 3) / 4;
  return (unsigned)(b < 1 ? 1 : (b > (1 << 20) ? (1 << 20) : b));
}

hipError_t launch_norm_rope(int dtype, int64_t N, const NormRope& nr, HeadRows q, HeadRows k,
                            const void* wq, const void* wk, const int32_t* pos, HeadRows qo, HeadRows ko,
                            hipStream_t st) {
  if (fast_heads(dtype, nr, {q, k, qo, ko}, {wq, wk})) {
    const RowsLaunch a = {N, nr, q, k, HeadRows{}, wq, wk, pos, qo, ko, PagedBatch{}, nullptr, nullptr, false, st};
    return dtype == kBF16 ? launch_rows_fast<uint16_t>(a) : launch_rows_fast<float>(a);
  }
  const unsigned blocks = wave_blocks(N * (q.H + k.H));
  if (dtype == kBF16)
    hipLaunchKernelGGL((norm_rope_generic<uint16_t>), dim3(blocks), dim3(256), 0, st, (int)N, nr, q, k,
                       (const uint16_t*)wq, (const uint16_t*)wk, pos, qo, ko);
  else
    hipLaunchKernelGGL((norm_rope_generic<float>), dim3(blocks), dim3(256), 0, st, (int)N, nr, q, k,
                       (const float*)wq, (const float*)wk, pos, qo, ko);
  return hipGetLastError();
}

// Two blocks of 8 waves on every compute unit: 12205 tokens of 48 heads of 128
// take 147 / 89 / 80 / 84 / 90 us (with the sum over blocks) for 128 / 256 / 512 /
// 1024 / 2048 blocks, 2000 tokens 31 / 23 / 22 / 29 / 40.  And a wave for every
// pass of a token at least: of float32 heads of 256 a wave covers two, a block 16
// (this counts for one token, and past 8192 heads).
int norm_rope_backward_blocks(int64_t N, int64_t heads) {
  const int64_t even = (N * heads + 31) / 32, b = even < 512 ? even : 512;
  const int64_t least = (heads + 2 * kBackWaves - 1) / (2 * kBackWaves);
  return (int)(b > least ? b : least);
}

hipError_t launch_norm_rope_backward(int dtype, int64_t N, const NormRope& nr, HeadRows q, HeadRows k,
                                     const void* wq, const void* wk, const int32_t* pos, HeadRows gq,
                                     HeadRows gk, HeadRows gqi, HeadRows gki, float* gwq, float* gwk,
                                     float* ws, hipStream_t st) {
  const int blocks = N ? norm_rope_backward_blocks(N, q.H + k.H) : 0;
  float* stage = (gwq || gwk) ? ws : nullptr;
  if (blocks && fast_heads(dtype, nr, {q, k, gq, gk, gqi, gki}, {wq, wk})) {
    const BackLaunch a = {N, nr, q, k, wq, wk, pos, gq, gk, gqi, gki, stage, blocks, st};
    const hipError_t e = dtype == kBF16 ? launch_back_fast<uint16_t>(a) : launch_back_fast<float>(a);
    if (e != hipSuccess) return e;
  } else if (blocks && dtype == kBF16)
    hipLaunchKernelGGL((norm_rope_backward_generic<uint16_t>), dim3(blocks), dim3(256), 0, st, (int)N, nr,
                       q, k, (const uint16_t*)wq, (const uint16_t*)wk, pos, gq, gk, gqi, gki, stage);
  else if (blocks)
    hipLaunchKernelGGL((norm_rope_backward_generic<float>), dim3(blocks), dim3(256), 0, st, (int)N, nr, q,
                       k, (const float*)wq, (const float*)wk, pos, gq, gk, gqi, gki, stage);
  if (gwq || gwk)
    hipLaunchKernelGGL(weight_grad_sum, dim3((nr.D + 15) / 16, 2), dim3(256), 0, st, stage, blocks, nr.D,
                       gwq, gwk);
  return hipGetLastError();
}

hipError_t launch_kv_append(int dtype, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k,
                            HeadRows v, const void* wq, const void* wk, void* Kc, void* Vc, HeadRows qo,
                            hipStream_t st) {
  if (fast_heads(dtype, nr, {q, k, v, qo}, {wq, wk, Kc, Vc})) {
    const RowsLaunch a = {pb.N, nr, q, k, v, wq, wk, nullptr, qo, HeadRows{}, pb, Kc, Vc, true, st};
    return dtype == kBF16 ? launch_rows_fast<uint16_t>(a) : launch_rows_fast<float>(a);
  }
  const unsigned blocks = wave_blocks((int64_t)pb.N * (q.H + 2 * k.H));
  if (dtype == kBF16)
    hipLaunchKernelGGL((kv_append_generic<uint16_t>), dim3(blocks), dim3(256), 0, st, pb, nr, q, k, v,
                       (const uint16_t*)wq, (const uint16_t*)wk, (uint16_t*)Kc, (uint16_t*)Vc, qo);
  else
    hipLaunchKernelGGL((kv_append_generic<float>), dim3(blocks), dim3(256), 0, st, pb, nr, q, k, v,
                       (const float*)wq, (const float*)wk, (float*)Kc, (float*)Vc, qo);
  return hipGetLastError();
}

}  // namespace ssn
