// dK and dV of the differential attention, bf16: four waves a block, 32 keys a wave, two blocks a CU, 32 queries a step.
//
//   dP' = V dO^T - delta_1,  S_m = K_m Q_m^T,  P_m = exp2(c S_m - lse_m),  then as operands in bf16 (to nearest even)
//   dV += (P_1 - lambda P_2) dO,  dK_1 += (P_1 dP') Q_1,  dK_2 += (P_2 (delta_2 - delta_1 - dP')) Q_2
// with scale and lambda left to the end.  dP' has delta_1 as its starting value, and its sum is rounded once in 32 bits.
//
// Bound by the two kinds of work of a SIMD, which hardly overlap: with dQ's blocks in the launch, matrix products keep it busy for 0.54 of the cycles and
// vector instructions for 0.50 (0.57 exponents a product, plain attention has 0.25 and 0.33; half of a step's vector work has no product beside it), at 1.87 GHz and
// 1,275 W of the card's 1,400.  The plain attention's kernels, at the same clock: 0.73 and 0.31, 0.78 and 0.37.  Two waves a SIMD leave a lane 256 registers: 128 hold dK and dV, 32
// K; with V's 32 as well the rest spills (11 ms), so V waits in LDS, where reading it takes less time than the products that use it.  One
// wave a SIMD with everything in registers is slower though it reads LDS less (48 keys a wave: 6.6 ms against 5.9), because a wave by itself
// overlaps little of its exponents and roundings with its products; a block of eight waves sharing a tile waits at its barriers (6.2).
// 62,400 x 12 heads, 8 groups: dK, dV and dQ in one launch 10.6 ms, 1.05 PFLOP/s of 7 products of 256 operations a pair of rows (plain attention's
// backward executes 1.3 on the same card).
#pragma once

#include "diff_attn.h"

namespace moga {

struct DiffKeySweep {
  static constexpr int NC = 2, kKeys = 16 * NC, kRows = 4 * kKeys;
  typedef DiffTiles<unsigned short, 128, true, 1, 2> Tiles;
  struct Lds {
    Tiles::Lds tiles;
    __attribute__((aligned(1024))) unsigned short v[kRows * kHeadDim];
  };
  bf16x8_t kf[NC][4];
  floatx4_t dk[8][NC], dv[8][NC];
  float c, lam;
  unsigned v_at;   // the lane's address of the wave's first 16 values' rows
  Tiles tiles;

  // The wave's own rows of V: operands of dP, which 32 registers more would be needed for, so they wait in LDS.
  __device__ __forceinline__ void keep_values(Lds& lds, const bf16x8_t (&vf)[NC][4]) {
    const int lane = threadIdx.x & 63, row = (threadIdx.x >> 6) * kKeys + (lane & 15);
    v_at = (unsigned)(uintptr_t)&lds.v[0] + row * 64 + (((lane >> 4) ^ lds_swizzle(row & 31)) << 4);
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) *(bf16x8_t __attribute__((address_space(3)))*)(uintptr_t)value_at(k, kb) = vf[k][kb];
  }
  // rows 16 .. 31 have the other swizzle bit
  __device__ __forceinline__ unsigned value_at(int k, int kb) const { return (v_at ^ (k << 4)) + k * 1024 + kb * kQuarterBytes<kRows>; }

  template <bool MASK>
  __device__ __forceinline__ void step(int left) {
    constexpr int kKeep = 0x2 | 0x4 | 0x400;   // vector, scalar and transcendental instructions
    const int g = (threadIdx.x & 63) >> 4;
    const unsigned nat = in_register(tiles.n_[0] + tiles.off);
    const unsigned tr[2] = {in_register(tiles.t_[0][0] + tiles.off), in_register(tiles.t_[0][1] + tiles.off)};
    constexpr unsigned kB = Tiles::kSlots * Tiles::kTile;   // from Q to dO
    floatx4_t s[2][NC], dp[2][NC], lse[2], by;
    uintx4_t pa[NC], p1[NC], p2[NC];
    bf16x8_t fd[2][4], fv[NC][4], fq[2][4], ft[16];
    auto load_d = [&](int kb) {   // dO rows of both operands, V
#pragma unroll
      for (int t = 0; t < 2; ++t) fd[t][kb] = read_nat<32>(nat + kB, t, kb);
#pragma unroll
      for (int k = 0; k < NC; ++k) fv[k][kb] = lds_read_b128(value_at(k, kb));
    };
    auto load_q = [&](int f) { fq[f >> 2][f & 3] = read_nat<32>(nat, f >> 2, f & 3); };
    auto load_t = [&](int f) { ft[f] = read_tr<32>(tr, (f & 1 ? 0 : kB), f >> 1); };
    load_d(0);
#pragma unroll
    for (int t = 0; t < 2; ++t) {   // dP - delta_1
      const floatx4_t d = tiles.rows(2, 8 * g + 4 * t);
#pragma unroll
      for (int k = 0; k < NC; ++k) dp[t][k] = d;
    }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      __builtin_amdgcn_sched_barrier(kKeep);
      if (kb < 3) load_d(kb + 1);
      else load_q(0), load_q(1);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < NC; ++k) dp[t][k] = mfma16(fd[t][kb], fv[k][kb], dp[t][k]);
    }
    auto scores = [&](int t, int kb) {
#pragma unroll
      for (int k = 0; k < NC; ++k) s[kb >> 1][k] = mfma16(fq[t][kb], kf[k][kb], (kb & 1) == 0 ? floatx4_t{0.f, 0.f, 0.f, 0.f} : s[kb >> 1][k]);
    };
    auto work = [&](const floatx4_t (&w)[2][NC], int t) {
      floatx4_t p[2][NC];
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int m = 0; m < 2; ++m) p[m][k][i] = fast_exp2(fmaf(w[m][k][i], c, -lse[m][i]));
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          float x[2], y[2], z[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[e] = fmaf(-lam, p[1][k][i + e], p[0][k][i + e]);
            y[e] = p[0][k][i + e] * dp[t][k][i + e];
            z[e] = p[1][k][i + e] * (by[i + e] - dp[t][k][i + e]);
          }
          pa[k][2 * t + (i >> 1)] = pack_bf16x2(x[0], x[1]);
          p1[k][2 * t + (i >> 1)] = pack_bf16x2(y[0], y[1]);
          p2[k][2 * t + (i >> 1)] = pack_bf16x2(z[0], z[1]);
        }
    };
    auto constants = [&](int t) {
#pragma unroll
      for (int m = 0; m < 2; ++m) lse[m] = tiles.rows(m, 8 * g + 4 * t);
      by = tiles.rows(3, 8 * g + 4 * t);
      if (MASK)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (8 * g + 4 * t + i >= left) lse[0][i] = lse[1][i] = INFINITY;
    };
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      __builtin_amdgcn_sched_barrier(kKeep);
      load_q(kb + 2);
      scores(0, kb);
    }
    constants(0);
    floatx4_t w[2][NC];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int k = 0; k < NC; ++k) w[m][k] = s[m][k];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      if (kb < 2) load_q(kb + 6);
      else load_t(kb - 2);
      scores(1, kb);
    }
    work(w, 0);
    __builtin_amdgcn_sched_barrier(0);
    constants(1);
    work(s, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < 16; ++f) {
      __builtin_amdgcn_sched_barrier(kKeep);
      if (f < 14) load_t(f + 2);
      const int dt = f >> 1;
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        if (f & 1) dk[dt][k] = mfma16(ft[f], __builtin_bit_cast(bf16x8_t, dt < 4 ? p1[k] : p2[k]), dk[dt][k]);
        else dv[dt][k] = mfma16(ft[f], __builtin_bit_cast(bf16x8_t, pa[k]), dv[dt][k]);
      }
    }
  }

  // Tile 0 is ready.
  __device__ __forceinline__ void sweep(int n) {
    const int full = n >> 5;
    for (int s = 0; s < full; ++s) {
      if (s > 0) tiles.ready(s);
      step<false>(32);
    }
    if (n & 31) {
      if (full > 0) tiles.ready(full);
      step<true>(n & 31);
    }
  }
};

}  // namespace moga
