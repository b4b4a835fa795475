// Norms of heads with the position rotation, forward and backward, and the
// serving form that writes keys and values into a paged cache.
//
// A head x of D values at position p, in float32:
//   r = (mean(x^2) + eps)^-1/2,  n = x r w,  y = rot_p(n)
// and for g = rot_p^T(dL/dy), h = g w:
//   dL/dx = r (h - x r mean(h x r)),   dL/dw = sum over rows of g x r
#include "attn_device.h"
#include "ssn_launch.h"

namespace ssn {

__global__ __launch_bounds__(256) void rope_table_kernel(float* __restrict__ table, int64_t P, int half,
                                                         double log_theta) {
  const int64_t n = P * half;
  for (int64_t e = blockIdx.x * (int64_t)256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
    const int64_t p = e / half;
    const int i = (int)(e - p * half);
    double s, c;
    sincos((double)p * exp(-log_theta * i / half), &s, &c);
    table[p * 2 * half + i] = (float)c;
    table[p * 2 * half + half + i] = (float)s;
  }
}

hipError_t launch_rope_table(int64_t P, int64_t R, double theta, float* table, hipStream_t st) {
  const int64_t n = P * (R / 2), blocks = (n + 255) / 256;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)(blocks > 65536 ? 65536 : blocks)), dim3(256), 0, st,
                     table, P, (int)(R / 2), log(theta));
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

static unsigned wave_blocks(int64_t waves) {
  const int64_t b = (waves + 3) / 4;
  return (unsigned)(b < 1 ? 1 : (b > (1 << 20) ? (1 << 20) : b));
}

hipError_t launch_norm_rope(int dtype, int64_t N, const NormRope& nr, HeadRows q, HeadRows k,
                            const void* wq, const void* wk, const int32_t* pos, HeadRows qo, HeadRows ko,
                            hipStream_t st) {
  const unsigned blocks = wave_blocks(N * (q.H + k.H));
  if (dtype == kBF16)
    hipLaunchKernelGGL((norm_rope_generic<uint16_t>), dim3(blocks), dim3(256), 0, st, (int)N, nr, q, k,
                       (const uint16_t*)wq, (const uint16_t*)wk, pos, qo, ko);
  else
    hipLaunchKernelGGL((norm_rope_generic<float>), dim3(blocks), dim3(256), 0, st, (int)N, nr, q, k,
                       (const float*)wq, (const float*)wk, pos, qo, ko);
  return hipGetLastError();
}

int norm_rope_backward_blocks(int64_t N, int64_t heads) {
  const int64_t b = (N * heads + 31) / 32;      // 8 heads a wave at least
  return (int)(b < 1 ? 1 : (b > 2048 ? 2048 : b));
}

hipError_t launch_norm_rope_backward(int dtype, int64_t N, const NormRope& nr, HeadRows q, HeadRows k,
                                     const void* wq, const void* wk, const int32_t* pos, HeadRows gq,
                                     HeadRows gk, HeadRows gqi, HeadRows gki, float* gwq, float* gwk,
                                     float* ws, hipStream_t st) {
  const int blocks = N ? norm_rope_backward_blocks(N, q.H + k.H) : 0;
  float* stage = (gwq || gwk) ? ws : nullptr;
  if (blocks && dtype == kBF16)
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
