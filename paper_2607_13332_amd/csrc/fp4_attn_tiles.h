// Attention of many rows over a 4-bit cache: a block of 4 waves owns a tile of rows
// of one sequence and key head (64 QB rows, 16 QB to a wave) and walks the keys the
// tile sees, 64 (or 32) at a time.  The codes of the tile after the next are on their
// way to registers, those of the next one become bf16 in LDS, double buffered, while
// this one's products run: each key is converted once for all the rows of a tile.
//
// What bounds it: the compute.  A prompt of 4096 tokens (40 / 8 heads of 128, bf16)
// takes 160 us, 1075 TFLOP/s where a large matrix product reaches 1230 to 1370, one of
// 8192 574, 1197 (over a bf16 cache 171 and 680: a quarter of the bytes saves more than
// the conversions cost).  The matrix cores are busy 46 % of the time, the vector units
// about as long, and the two hardly overlap.  Measured and not kept: the next tile's
// codes to LDS after the first half's scores (+4 %), in two parts (+1 %); blocks of 8
// waves and 384 rows whose halves take turns, barriers between, at products and
// exponentials (195 us, 218 without the turns).
//
// bf16 probabilities are rounded once for the product with V (2^-8 of each at most), as
// over a bf16 cache.  What the rounding leaves as a second product, as the rows kernel
// has it: prompts of 300 / 1024 / 2048 / 4096 tokens take 19 / 29 / 69 / 218 us with it
// and 18.5 / 26 / 55 / 160 without, 512 tokens over 32768 keys 382 and 279, 517 beside 31
// single ones 145 and 119.  The outputs' error against float64 is 0.0022 to 0.0023, 0.0016
// with it, which is their own rounding.  Float32 ones go in three parts, against one of K and V: prompts of
// 300 to 1024 tokens (16 heads of 64) 31 us where float32 products over a float32 cache
// take 70.
#pragma once

#include "attn_tiles.h"
#include "fp4_attn_mma.h"

namespace ssn {

template <int DT>
constexpr int fp4_tile_keys() { return DT <= 128 ? 64 : 32; }
template <int DT>
constexpr int fp4_tiles_lds() { return 4 * fp4_tile_keys<DT>() * DT * 2; }

template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void fp4_tiles_block(const Fp4AttnArgs& fa, const AttnPart& part, int few,
                                                const TileCount& count, int id, char* mem) {
  using Tag = OverFp4<T>;
  using M = Mma<Tag>;
  constexpr int RB = DT * 2, TK = fp4_tile_keys<DT>(), NC = DT / 32, PARTS = M::kTilesParts, BM = 64 * QB;
  // keys whose scores are held at a time
  constexpr int SK = 32, NKB = SK / 16;
  // A thread fetches a unit of UW dwords of codes, UE elements of one group.
  constexpr int UPK = 256 / TK, UE = DT / UPK, UW = UE / 8, KPW = kWave / UPK;
  const AttnArgs& a = fa.a;
  char(*lds)[2][TK * RB] = (char(*)[2][TK * RB])mem;      // [buffer][K, V]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kh = id % a.Hk, rest = id / a.Hk;
  if (count.total <= 0) return;
  const int range = rest / count.total;
  int b, tile;
  if (range >= part.ranges ||
      !count.find(a.pb, a.G, BM, few, balanced_order(rest % count.total, count.total, a.Hk), b, tile))
    return;
  const Sequence sq = sequence_of(a.pb, b);
  const int n = sq.s1 - sq.s0, rows = n * a.G, r0 = tile * BM;
  const int before = sq.len - n;                           // position of the sequence's token 0
  const int last = r0 + BM < rows ? r0 + BM - 1 : rows - 1;
  const int keys = before + last / a.G + 1;                // that the tile sees
  const int ranges = key_ranges(keys, part.chunk);
  if (range >= ranges) return;

  const int groups = a.D / kFp4Group;
  int row[QB], seen[QB];
  u32x4 qf[QB][NC][M::kQueries];
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    row[q] = r0 + wave * (16 * QB) + q * 16 + (lane & 15);
    const int r = row[q] < rows ? row[q] : rows - 1, token = r / a.G;
    seen[q] = before + token;
    const T* p = (const T*)a.Q + (sq.s0 + token) * a.ldq + (int64_t)(kh * a.G + r % a.G) * a.D;
#pragma unroll
    for (int ch = 0; ch < NC; ++ch) {
      const int e = 32 * ch + 8 * (lane >> 4);
      QueryChunk<T> x;
      x.load(p + e, a.scale != 0.f && (EXACT || e < a.D));
      x.parts(sign_bits<T>(a.scale), qf[q][ch]);
    }
  }
  // a scale of zero: zero queries, any other scale
  const float c = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * kLog2e;
  const int wave_last = r0 + (wave + 1) * (16 * QB) - 1;
  const int seen_hi = before + (wave_last < rows ? wave_last : rows - 1) / a.G;

  const int t0 = range * (part.chunk / TK);
  const int all = (keys + TK - 1) / TK, t1 = all < t0 + part.chunk / TK ? all : t0 + part.chunk / TK;

  // This thread's key of a tile, and the unit of its codes.  Keys past the last
  // repeat it (their scores are masked).
  const int unit = lane / KPW, e0 = unit * UE, key = wave * KPW + (lane & (KPW - 1));
  const int v_row = (key & ~15) + value_row(key & 15);
  typedef uint32_t piece __attribute__((ext_vector_type(UW)));
  piece kreg = {}, vreg = {};
  uint32_t ks = 0, vs = 0;
  Slot slot = {0, 0};
  auto find = [&](int t) { slot = find_slot(a.pb, b, t * TK + key < keys ? t * TK + key : keys - 1); };
  auto fetch = [&]() {
    const int64_t row = slot_row(a.pb, slot, a.Hk, kh), c = row * (a.D / 2) + e0 / 2, s = row * groups + e0 / kFp4Group;
    if (EXACT || e0 < a.D) {
      kreg = *(const piece*)((const uint8_t*)a.Kc + c);
      vreg = *(const piece*)((const uint8_t*)a.Vc + c);
      ks = fa.Ks[s];
      vs = fa.Vs[s];
    }
  };
  auto put_keys = [&](int buf) {
#pragma unroll
    for (int j = 0; j < UW; ++j)
      *(u32x4*)(&lds[buf][0][key * RB + (((uint32_t)(unit * UW + j) ^ swizzle_keys<RB>(key)) << 4)]) =
          fp4_bf16x8(kreg[j], fp4_scale(ks));
  };
  auto put_values = [&](int buf) {
#pragma unroll
    for (int j = 0; j < UW; ++j)
      *(u32x4*)(&lds[buf][1][v_row * RB + (((uint32_t)(unit * UW + j) ^ swizzle_values<RB>(v_row)) << 4)]) =
          fp4_bf16x8(vreg[j], fp4_scale(vs));
  };

  const uint32_t vb[1] = {value_base<RB>(lane)};
  const uint32_t kb0 = (lane & 15) * RB + (((uint32_t)(lane >> 4) ^ swizzle_keys<RB>(lane & 15)) << 4);

  RowState<DT / 16, QB> rs;
  rs.clear();
  uint32_t odd = 0;
  // before tile t: its keys and values in LDS, tile t + 1's codes in registers,
  // tile t + 2's slots
  if (t0 < t1) {
    find(t0);
    fetch();
    put_keys(0);
    put_values(0);
    if (t0 + 1 < t1) {
      find(t0 + 1);
      fetch();
    }
    if (t0 + 2 < t1) find(t0 + 2);
  }
  auto stage = [&](int t) {
    // the codes of tile t + 1 to LDS, where everyone is done with tile t - 1
    if (t + 1 < t1) {
      put_keys((t + 1 - t0) & 1);
      put_values((t + 1 - t0) & 1);
    }
    if (t + 2 < t1) fetch();
    if (t + 3 < t1) find(t + 3);
  };
  // The widest tiles, and those of narrow heads, ask for the matrix cores first
  // (s_setprio), so that of a SIMD's two waves one multiplies while the other
  // exponentiates: 177 -> 162 us for a prompt of 4096 tokens (40 / 8 heads of 128), 92
  // -> 89 with 32 / 8 heads of 64; 128 rows of heads of 128 lose 5 %, heads of 256 20.
  constexpr bool kFirst = QB == 3 || (QB == 2 && DT == 64);
  // Where a tile's scores are held at once its next codes go to LDS after its products
  // (2048 tokens, 8 / 2 heads of 256: 78 -> 71 us), else before (4096 tokens of heads
  // of 128: 162 us, 167 after the first half's products).
  constexpr bool kLate = TK == SK;
  auto scores = [&](const char* kl, f32x4 (&s)[NKB][QB]) {
#pragma unroll
    for (int k = 0; k < NKB; ++k) {
#pragma unroll
      for (int q = 0; q < QB; ++q) s[k][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ch = 0; ch < NC; ++ch) {
        const u32x4 kf = *(const u32x4*)(kl + (kb0 ^ (uint32_t)(ch * 64)) + k * 16 * RB);
#pragma unroll
        for (int q = 0; q < QB; ++q)
#pragma unroll
          for (int m = M::kQueries - 1; m >= 0; --m) s[k][q] = M::mma(kf, qf[q][ch][m], s[k][q]);
      }
    }
  };
  // Tiles that every row of the block sees, then the others.
  const int open = (before + r0 / a.G + 1) / TK, t_open = open < t0 ? t0 : (open < t1 ? open : t1);
  int t = t0;
  for (; t < t_open; ++t) {
    __syncthreads();
    const char *kl = lds[(t - t0) & 1][0], *vl = lds[(t - t0) & 1][1];
    if constexpr (!kLate) stage(t);
#pragma unroll
    for (int u = 0; u < TK; u += SK) {
      f32x4 s[NKB][QB];
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
      scores(kl + u * RB, s);
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(0);
      u32x4 p[PARTS][NKB / 2][QB];
      softmax_step<Tag, PARTS>(s, rs, c, p);
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
      weigh<Tag, RB, false>(vl + u * RB, vb, p, rs, odd);
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(0);
    }
    if constexpr (kLate) stage(t);
  }
  for (; t < t1; ++t) {
    __syncthreads();
    const char *kl = lds[(t - t0) & 1][0], *vl = lds[(t - t0) & 1][1];
    stage(t);
#pragma unroll 1
    for (int u = 0; u < TK; u += SK) {
      const int k0 = t * TK + u;
      if (k0 > seen_hi) break;
      f32x4 s[NKB][QB];
      scores(kl + u * RB, s);
#pragma unroll
      for (int q = 0; q < QB; ++q)
#pragma unroll
        for (int k = 0; k < NKB; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * k + 4 * (lane >> 4) + i > seen[q] - k0) s[k][q][i] = kNegInf;
      u32x4 p[PARTS][NKB / 2][QB];
      softmax_step<Tag, PARTS>(s, rs, c, p);
      weigh<Tag, RB, true>(vl + u * RB, vb, p, rs, odd);
    }
  }
  if (__any(odd != 0)) {
    // the keys of the masked tiles
#pragma unroll 1
    for (int k = t_open * TK; k < t1 * TK && k <= seen_hi; ++k) {
      bool sees[QB];
#pragma unroll
      for (int q = 0; q < QB; ++q) sees[q] = k <= seen[q];
      add_not_finite_groups(fa.Vs + (int64_t)cache_row(a.pb, b, a.Hk, kh, k) * groups, a.D, sees, rs);
    }
  }
  finish_rows<T, DT, QB, EXACT>(a, part, rs, row, seen, rows, sq.s0, kh, range, -1, ranges == 1, c, lane);
}

}  // namespace ssn
