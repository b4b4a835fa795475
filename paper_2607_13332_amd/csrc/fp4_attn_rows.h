// Attention of few rows over a 4-bit cache: a block of 4 waves owns a range of the
// keys of one sequence and key head; its waves take the range's tiles of 32 keys in
// turn, all with the same 16 QB rows, and join their results in LDS at the end.
//
// Keys are A operands as they come: a lane's 16 bytes are one group of its key, and a
// product takes the elements 8 ch .. 8 ch + 7 of every lane's group, which the queries
// are ordered to match.  Values become bf16 on their way to the wave's part of LDS and
// are read transposed.  A lane has the same key of both, so that their addresses are
// worked out once.
//
// What bounds it: memory, and for short caches the waits at a block's beginning and end.
// 64 single tokens over caches of 1 to 4096 keys (8 heads of 128) take 37 us (3.9 TB/s)
// and their join 6, four over 100000 to 131072 100 (5.6 TB/s; a large copy moves 5.1)
// and 8; with the loads alone, nothing computed, 36 and 88.  The vector units issue
// half of the time, the matrix cores a fifth; registers for four blocks of a compute
// unit instead of three gain nothing.  Kept on the way, the two times in sum: as first
// built 56 / 132; loads without a condition, tiles of 32 keys and three blocks 44 / 109;
// one address for keys and values, queries in LDS, one exchange at the end 43 / 108.
//
// Probabilities go in the parts of attn_rows.h: two for bf16 (2^-16 of each), three for
// float32 (all its bits).
#pragma once

#include "attn_rows.h"
#include "fp4_attn_mma.h"

namespace ssn {

constexpr int kFp4Keys = 32;           // of a wave's tile
// LDS: a wave's values, 32 keys at a time, and at the end its O; m and l of the
// waves; the block's queries.
template <int DT, int QB>
constexpr int fp4_wave_lds() {
  const int values = 32 * DT * 2, o = DT / 16 * QB * kWave * 16;
  return values > o ? values : o;
}
template <int DT, int QB>
constexpr int fp4_join_lds() { return 4 * fp4_wave_lds<DT, QB>() + 4 * QB * 2 * kWave * 4; }
template <typename T, int DT, int QB>
constexpr int fp4_rows_lds() { return fp4_join_lds<DT, QB>() + QB * (DT / 32) * Mma<OverFp4<T>>::kQueries * kWave * 16; }

// The waves' results, joined and stored by all of them: a wave takes a quarter of the
// head.  With M the largest m, O = sum exp2((m - M) c) O_w / sum exp2((m - M) c) l_w,
// in the waves' order.
template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void fp4_finish(const AttnArgs& a, const AttnPart& part, const RowState<DT / 16, QB>& rs,
                                           char* lds, const int (&seen)[QB], int rows, int s0, int kh, int range,
                                           int64_t stage0, bool whole, float c, int lane, int wave) {
  constexpr int DT16 = DT / 16, kO = fp4_wave_lds<DT, QB>();
  float(*ml)[QB][2][kWave] = (float(*)[QB][2][kWave])(lds + 4 * kO);
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    ml[wave][q][0][lane] = rs.m[q];
    ml[wave][q][1][lane] = column_sum(rs.l[q]);
#pragma unroll
    for (int d = 0; d < DT16; ++d) *(f32x4*)(lds + wave * kO + ((d * QB + q) * kWave + lane) * 16) = rs.o[d][q];
  }
  __syncthreads();
  const int h4 = 4 * (lane >> 4);
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    const int row = q * 16 + (lane & 15);
    if (row >= rows) continue;
    float m[4], top = kNegInf, l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      m[w] = ml[w][q][0][lane];
      top = fmaxf(top, m[w]);
    }
    const float base = top == kNegInf ? 0.f : top;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      m[w] = __builtin_amdgcn_exp2f((m[w] - base) * c);
      l += ml[w][q][1][lane] * m[w];
    }
    const int token = s0 + row / a.G, head = kh * a.G + row % a.G;
    // 0 / 0 where every score a row sees is -inf; a row that sees nothing is zero
    const float inv = seen[q] < 0 ? 0.f : 1.f / l;
    T* out = (T*)a.O + token * a.ldo + (int64_t)head * a.D;
    const int64_t to = range * part.stage_rows + stage0 + row;
#pragma unroll
    for (int i = 0; i < DT16 / 4; ++i) {
      const int d = wave * (DT16 / 4) + i;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) o += *(const f32x4*)(lds + w * kO + ((d * QB + q) * kWave + lane) * 16) * m[w];
      if (!EXACT && 16 * d + h4 >= a.D) continue;
      if (whole) store4(out + 16 * d + h4, o * inv);
      else *(f32x4*)(part.o + to * a.D + 16 * d + h4) = o;
    }
    if (wave == 0 && lane < 16) {
      if (!whole) {
        part.ml[2 * to] = top * c;
        part.ml[2 * to + 1] = l;
      } else if (a.lse) {
        a.lse[(int64_t)token * a.Hq + head] = seen[q] < 0 ? kNegInf : (top * c + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
      }
    }
  }
}

template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void fp4_rows_block(const Fp4AttnArgs& fa, const AttnPart& part, int few, int id, char* lds) {
  using Tag = OverFp4<T>;
  using M = Mma<Tag>;
  constexpr int RB = DT * 2, TK = kFp4Keys, NKB = TK / 16, NC = DT / 32, DT16 = DT / 16, PARTS = M::kRowsParts;
  // A key's lanes 16 g + its number hold the g-th quarter of its head, UW dwords
  // of codes and SC scales: 16 bytes of one group where the head has 128 elements.
  constexpr int UE = DT / 4, UW = UE / 8, SC = UE > kFp4Group ? UE / kFp4Group : 1;
  const AttnArgs& a = fa.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kh = id % a.Hk, rest = id / a.Hk, b = rest % a.pb.B, range = rest / a.pb.B;
  const Sequence sq = sequence_of(a.pb, b);
  const int n = sq.s1 - sq.s0, rows = n * a.G, keys = sq.len;
  if (rows == 0 || rows > few) return;
  const int ranges = key_ranges(keys, part.chunk);
  if (range >= ranges) return;
  const int before = sq.len - n, D = EXACT ? DT : a.D, groups = D / kFp4Group;
  const int k_begin = range * part.chunk, k_end = range_end(k_begin, part.chunk, keys);
  const int g = lane >> 4, e0 = g * UE;

  const float c = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * kLog2e;

  // The queries are the same in all waves: in LDS, which leaves 16 registers and more
  // to a wave.  Their loads go first and are waited for last.
  constexpr int QC = (NC + 3) / 4;
  u32x4(*ql)[NC][M::kQueries][kWave] = (u32x4(*)[NC][M::kQueries][kWave])(lds + fp4_join_lds<DT, QB>());
  QueryChunk<T> raw[QB][QC];
  int seen[QB];
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    const int row = q * 16 + (lane & 15), r = row < rows ? row : rows - 1, token = r / a.G;
    seen[q] = before + token;
    const T* p = (const T*)a.Q + (sq.s0 + token) * a.ldq + (int64_t)(kh * a.G + r % a.G) * a.D;
#pragma unroll
    for (int i = 0; i < QC; ++i) {
      const int ch = 4 * i + wave, e = e0 + 8 * ch;
      raw[q][i].load(p + e, a.scale != 0.f && ch < NC && (EXACT || e < a.D));
    }
  }

  char* vl = lds + wave * fp4_wave_lds<DT, QB>();
  uint32_t kreg[NKB][UW], vreg[NKB][UW];
  uint8_t ks[NKB][SC], vs[NKB][SC];
  auto rows_of = [&](int t) {
    const int ahead = keys - 1 - t, key = (lane & (TK - 1));     // (t + key may pass 2^31)
    return find_slot(a.pb, b, key < ahead ? t + key : keys - 1);
  };
  // where the lane's part of a key's codes and scales begins, of keys and of values
  uint32_t lane_c = e0 / 2, lane_s = e0 / kFp4Group;
  uint64_t at_c[NKB], at_s[NKB];
  auto place = [&](const Slot& slot) {
    const uint32_t mine = slot_row(a.pb, slot, a.Hk, kh);
#pragma unroll
    for (int k = 0; k < NKB; ++k) {
      const uint32_t r = (uint32_t)__shfl((int)mine, 16 * k + (lane & 15), kWave);
      at_c[k] = (uint64_t)r * (uint32_t)(D / 2) + lane_c;
      at_s[k] = (uint64_t)r * (uint32_t)groups + lane_s;
    }
  };
  auto load = [&](const void* codes, const uint8_t* scales, int k, uint32_t (&w)[UW], uint8_t (&s)[SC]) {
    constexpr int V = UW < 4 ? UW : 4;
    typedef uint32_t piece __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int i = 0; i < UW; i += V) {
      piece x = {};
      if (EXACT || e0 + 8 * i < D) x = __builtin_nontemporal_load((const piece*)((const uint8_t*)codes + at_c[k] + 4 * i));
#pragma unroll
      for (int j = 0; j < V; ++j) w[i + j] = x[j];
    }
#pragma unroll
    for (int i = 0; i < SC; ++i) {
      s[i] = 0;
      if (EXACT || e0 + 32 * i < D) s[i] = scales[at_s[k] + i];
    }
  };
  const int v_row = value_row(lane & 15);
  uint32_t vb[1] = {value_base<RB>(lane)}, vw = v_row * RB + (((uint32_t)(g * NC) ^ swizzle_values<RB>(v_row)) << 4);

  int t = k_begin + wave * TK;
  uint32_t odd = 0;
  Slot next = {0, 0};
  if (t < k_end) {
    place(rows_of(t));
#pragma unroll
    for (int k = 0; k < NKB; ++k) load(a.Kc, fa.Ks, k, kreg[k], ks[k]);
#pragma unroll
    for (int k = 0; k < NKB; ++k) load(a.Vc, fa.Vs, k, vreg[k], vs[k]);
    next = rows_of(t + 4 * TK);
  }
#pragma unroll
  for (int q = 0; q < QB; ++q)
#pragma unroll
    for (int i = 0; i < QC; ++i) {
      u32x4 x[M::kQueries];
      raw[q][i].parts(sign_bits<T>(a.scale), x);
#pragma unroll
      for (int m = 0; m < M::kQueries; ++m)
        if (4 * i + wave < NC) ql[q][4 * i + wave][m][lane] = x[m];
    }
  __syncthreads();

  RowState<DT16, QB> rs;
  rs.clear();
  for (; t < k_end; t += 4 * TK) {
    // (opaque to the compiler, which would keep what follows from them, bases and LDS
    // addresses of every lane, in registers throughout)
    asm volatile("" : "+v"(vb[0]), "+v"(vw), "+v"(lane_c), "+v"(lane_s));
    const bool masked = t + TK - 1 > before;
    f32x4 s[NKB][QB];
#pragma unroll
    for (int k = 0; k < NKB; ++k) {
#pragma unroll
      for (int q = 0; q < QB; ++q) s[k][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ch = 0; ch < NC; ++ch) {
        const u32x4 kf = fp4_bf16x8(kreg[k][ch], fp4_scale(ks[k][8 * ch / kFp4Group]));
#pragma unroll
        for (int q = 0; q < QB; ++q)
#pragma unroll
          for (int m = M::kQueries - 1; m >= 0; --m) s[k][q] = M::mma(kf, ql[q][ch][m][lane], s[k][q]);
      }
    }
    // the next tile, past the end its last key over again: without a condition,
    // which would have every load waited for where the paths meet
    place(next);
#pragma unroll
    for (int k = 0; k < NKB; ++k) load(a.Kc, fa.Ks, k, kreg[k], ks[k]);
    next = rows_of(t + 8 * TK);
    if (masked) {
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        const int last = seen[q] - t - 4 * g;
#pragma unroll
        for (int k = 0; k < NKB; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * k + i > last) s[k][q][i] = kNegInf;
      }
    }
    u32x4 p[PARTS][NKB / 2][QB];
    softmax_step<Tag, PARTS>(s, rs, c, p);
    // 32 keys' values at a time through the wave's part of LDS
#pragma unroll
    for (int half = 0; half < NKB / 2; ++half) {
      wave_lds_order();
#pragma unroll
      for (int k = 2 * half; k < 2 * half + 2; ++k) {
#pragma unroll
        for (int ch = 0; ch < NC; ++ch)
          *(u32x4*)(vl + 16 * (k & 1) * RB + (vw ^ (uint32_t)(ch << 4))) =
              fp4_bf16x8(vreg[k][ch], fp4_scale(vs[k][8 * ch / kFp4Group]));
        load(a.Vc, fa.Vs, k, vreg[k], vs[k]);
      }
      wave_lds_order();
      u32x4 ph[PARTS][1][QB];
#pragma unroll
      for (int m = 0; m < PARTS; ++m)
#pragma unroll
        for (int q = 0; q < QB; ++q) ph[m][0][q] = p[m][half][q];
      if (masked) weigh<Tag, RB, true>(vl, vb, ph, rs, odd);
      else weigh<Tag, RB, false>(vl, vb, ph, rs, odd);
    }
  }
  if (__any(odd != 0)) {
    // the keys of this wave's masked tiles
#pragma unroll 1
    for (int k = k_begin + wave * TK; k < k_end; k += 4 * TK)
#pragma unroll 1
      for (int u = k; u < k + TK && u < k_end && k + TK - 1 > before; ++u) {
        bool sees[QB];
#pragma unroll
        for (int q = 0; q < QB; ++q) sees[q] = u <= seen[q];
        add_not_finite_groups(fa.Vs + (int64_t)cache_row(a.pb, b, a.Hk, kh, u) * groups, a.D, sees, rs);
      }
  }
  fp4_finish<T, DT, QB, EXACT>(a, part, rs, lds, seen, rows, sq.s0, kh, range, ((int64_t)b * a.Hk + kh) * (16 * QB),
                               ranges == 1, c, lane, wave);
}

}  // namespace ssn
