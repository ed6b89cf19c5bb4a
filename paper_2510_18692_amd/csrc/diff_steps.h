// The bf16 forward of the differential attention: 32 queries a wave in two columns of 16, 32 keys a step, two waves a SIMD.
//
// With a step's vector work all between its products, two waves overlap little: a step took the sum of its products' and its vector
// work's cycles.  Here the vector work of one group of products lies among the next ones; fragments are read two ahead, and only
// vector instructions may cross a group.  62,400 x 12 heads, 8 groups 4.5 -> 4.25 ms, 32,760 x 12, 8 groups 1.46 -> 1.27 (4.3 and 1.31 on another
// card; 1.11 PFLOP/s of 768 operations a pair, where plain attention's forward executes 1.3).  Bound by both kinds of work of a SIMD: matrix products 0.59 of the cycles,
// vector instructions 0.54 (two exponents for every three products, one for two in plain attention), at 1.82 GHz and 1,312 W of 1,400.  32 queries a wave: an
// accumulator of 16 more would not fit beside two maps' sums of V, and 16 would read every fragment for half the products.  A block of
// eight waves was slower (4.5 ms).
#pragma once

#include "diff_attn.h"

namespace moga {

constexpr int kVectorMayCross = 0x2 | 0x4 | 0x400;   // vector, scalar and transcendental instructions
constexpr int kAheadFrags = 2;

// Forward, a map at a time: while the matrix cores compute the scores of the next half step (the other map's, then the next 32 keys'), the vector
// units make the weights of this one; while they add V^T P^T, the scores become exponents and their maximum is taken.
//   S(s, 2), P(s, 1) | O_1, exponents (s, 2) | S(s + 1, 1), P(s, 2) | O_2, exponents (s + 1, 1)
struct DiffFwdSweep {
  static constexpr int NC = 2;
  typedef DiffTiles<unsigned short, 128, false, 2> Tiles;
  typedef floatx4_t Half[2][NC];   // scores or exponents: key 8 g + 4 t + i of column q
  bf16x8_t qf[NC][4];
  floatx4_t o[2][8][NC];
  float m[2][NC], l[2][NC], thresh[2][NC], mx[NC], c;
  bf16x8_t ahead[kAheadFrags];
  unsigned nat, tr[2];   // the lane's addresses: K rows of the tile whose scores come next, V transposed of the present one
  Tiles tiles;

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        m[k][q] = l[k][q] = 0.f;
        thresh[k][q] = -INFINITY;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[k][dt][q] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      }
  }
  template <bool MASK>
  __device__ __forceinline__ void exponents(int map, Half& x, int q, int left) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[t][q][i] = fmaf(x[t][q][i], c, -m[map][q]);
        if (MASK && 8 * g + 4 * t + i >= left) x[t][q][i] = -INFINITY;
      }
    mx[q] = column_max(x, q);
  }
  // The maximum is raised when a weight would exceed 2^8 only: rare after the first step.
  __device__ __forceinline__ void raise(int map, Half& x) {
    bool up = false;
#pragma unroll
    for (int q = 0; q < NC; ++q) up = up || mx[q] > thresh[map][q];
    if (__builtin_amdgcn_ballot_w64(up) == 0) return;
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      float all = fmaxf(mx[q], __shfl_xor(mx[q], 16, kWave));
      all = fmaxf(all, __shfl_xor(all, 32, kWave));
      const bool first = thresh[map][q] == -INFINITY;
      const float by = first ? (all == -INFINITY ? 0.f : all) : fmaxf(all, 0.f);
      const float alpha = first ? 0.f : fast_exp2(-by);
      if (all != -INFINITY) thresh[map][q] = 8.f;
      m[map][q] += by;
      l[map][q] *= alpha;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][q][i] -= by;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[map][dt][q] *= alpha;
    }
  }
  __device__ __forceinline__ bf16x8_t row_frag(int map, int f) const { return read_nat<32>(nat, f >> 1, 2 * map + (f & 1)); }   // f: (t, kb)

  // Scores of `map` of the tile at nat to `sn` (SCORES), weights of the other map from `x`, their weighted sum of V; then sn as exponents.
  // mid(): called two fragments before the end, where the next tile is waited for.  THEN: the scores after these are computed too (fragments
  // of map `after` are read ahead).
  template <bool SCORES, bool MASK, bool THEN, typename F>
  __device__ __forceinline__ void half(int map, Half& x, Half& sn, int left, F&& mid) {
    const int cur = SCORES ? map ^ 1 : map;
    bf16x8_t fr[12];
    unsigned pk[NC][4];
    auto load = [&](int f) {
      if (f < 4) fr[f] = row_frag(map, f);
      else if (f < 12) fr[f] = read_tr<32>(tr, 4 * Tiles::kTile, f - 4);
      else if (THEN) ahead[f - 12] = row_frag(map ^ 1, f - 12);
    };
    auto word = [&](int q, int w) {   // keys 8 g + 2 w and + 1; sums in 32 bits, before the weights are rounded to operands
      const float a = fast_exp2(x[w >> 1][q][2 * (w & 1)]), b = fast_exp2(x[w >> 1][q][2 * (w & 1) + 1]);
      l[cur][q] += a + b;
      pk[q][w] = pack_bf16x2(a, b);
    };
    if constexpr (SCORES) {
#pragma unroll
      for (int f = 0; f < kAheadFrags; ++f) fr[f] = ahead[f];
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        __builtin_amdgcn_sched_barrier(kVectorMayCross);
        load(f + kAheadFrags);
#pragma unroll
        for (int q = 0; q < NC; ++q)
          sn[f >> 1][q] = mfma16(fr[f], qf[q][2 * map + (f & 1)], (f & 1) == 0 ? floatx4_t{0.f, 0.f, 0.f, 0.f} : sn[f >> 1][q]);
#pragma unroll
        for (int q = 0; q < NC; ++q) word(q, f);
      }
    } else {
#pragma unroll
      for (int f = 4; f < 4 + kAheadFrags; ++f) load(f);
#pragma unroll
      for (int q = 0; q < NC; ++q)
#pragma unroll
        for (int w = 0; w < 4; ++w) word(q, w);
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8_t pf[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) pf[q] = __builtin_bit_cast(bf16x8_t, uintx4_t{pk[q][0], pk[q][1], pk[q][2], pk[q][3]});
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      if (dt == 8 - kAheadFrags) mid();
      __builtin_amdgcn_sched_barrier(kVectorMayCross);
      load(4 + dt + kAheadFrags);
      if (SCORES && (dt == 2 || dt == 4)) exponents<MASK>(map, sn, dt / 2 - 1, left);
#pragma unroll
      for (int q = 0; q < NC; ++q) o[cur][dt][q] = mfma16(fr[4 + dt], pf[q], o[cur][dt][q]);
    }
    if constexpr (SCORES) raise(map, sn);
  }

  __device__ __forceinline__ void next_tile(int s) {
    tiles.ready(s);
    nat = in_register(tiles.n_[0] + tiles.off);
  }
  __device__ __forceinline__ void value_tile(int s) {
#pragma unroll
    for (int p = 0; p < 2; ++p) tr[p] = in_register(tiles.t_[0][p] + (unsigned)(s & 3) * Tiles::kTile);
  }

  // Tile 0 is ready.  The last tile's scores are masked whether it is whole or not.
  __device__ __forceinline__ void sweep(int n) {
    const int steps = (n + 31) >> 5, left = n - 32 * (steps - 1);
    auto nothing = []() {};
    Half x, y;
    nat = in_register(tiles.n_[0] + tiles.off);
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      __builtin_amdgcn_sched_barrier(0);
      const bf16x8_t a = row_frag(0, f);
#pragma unroll
      for (int q = 0; q < NC; ++q) x[f >> 1][q] = mfma16(a, qf[q][f & 1], (f & 1) == 0 ? floatx4_t{0.f, 0.f, 0.f, 0.f} : x[f >> 1][q]);
    }
#pragma unroll
    for (int q = 0; q < NC; ++q) exponents<true>(0, x, q, min(n, 32));
    raise(0, x);
#pragma unroll
    for (int f = 0; f < kAheadFrags; ++f) ahead[f] = row_frag(1, f);
    int s = 0;
    for (; s < steps - 2; ++s) {   // tiles whose successor is not the last
      value_tile(s);
      half<true, false, true>(1, x, y, 32, [&]() { next_tile(s + 1); });
      half<true, false, true>(0, y, x, 32, nothing);
    }
    if (s < steps - 1) {
      value_tile(s);
      half<true, false, true>(1, x, y, 32, [&]() { next_tile(s + 1); });
      half<true, true, true>(0, y, x, left, nothing);
      ++s;
    }
    value_tile(s);
    half<true, true, false>(1, x, y, left, nothing);
    half<false, false, false>(1, y, x, 32, nothing);
  }
};

}  // namespace moga
