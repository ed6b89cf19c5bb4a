// dK and dV of the differential attention, bf16: four waves a block, one per SIMD, 48 keys a wave.
//
// A wave keeps 48 keys (K and V fragments) and their dK^T and dV^T, 288 registers, and sweeps the queries of its group, 32 a step, in LDS beside
// their row constants.  Per 16 queries (t = 0, 1) of a step: scores of both maps and dP, 24 products; from them
//   a = P_1 - lambda P_2, d_1 = P_1 (dP - delta_1), d_2 = P_2 (delta_2 - dP)        (dK_2 is multiplied by lambda at the end)
// and with 32 queries of a, d_1 and d_2 the 48 products of dV^T += dO^T a and dK_m^T += Q_m^T d_m.  A fragment read from LDS feeds three products.
//
// One wave has to fill both pipes: a product takes 16 cycles and leaves 12 of them to vector instructions, and a step has 96 products and
// some 1,200 cycles of vector work.  So the work of tile s lies between the products of tile s + 1 and its own last ones, a few vector
// instructions behind every product:
//   scores, dP (t = 0) of s + 1   |  a, d_1, d_2 of s, t = 1
//   dV, dK of s                   |  all of s + 1, t = 0
//   scores, dP (t = 1) of s + 1   |  P_1, P_2 of s + 1, t = 1
#pragma once

#include "diff_attn.h"

namespace moga {

struct DiffKeySweep {
  static constexpr int NC = 3, kKeys = 16 * NC, kWin = 2;   // kWin: fragments read ahead
  typedef DiffTiles<unsigned short, 128, true, 2> Tiles;
  struct Half { floatx4_t s[2][NC], dp[NC], rc[4]; };       // scores, then weights, and dP of 16 queries; their row constants
  struct Packed { uintx4_t a[NC], d1[NC], d2[NC]; };        // of 32 queries: t = 0 in words 0, 1

  bf16x8_t kf[NC][4], vf[NC][4], ahead[kWin];
  floatx4_t dk[8][NC], dv[8][NC];
  Half h0, h1;
  float c, lam;
  unsigned nat, tr[2];   // the lane's addresses: rows of the newer tile, transposed of the older
  Tiles tiles;

  __device__ __forceinline__ void load_rows(int t, Half& h) {
#pragma unroll
    for (int v = 0; v < 4; ++v) h.rc[v] = tiles.rows(v, 8 * ((threadIdx.x & 63) >> 4) + 4 * t);
  }
  // queries behind the last: weights of zero
  __device__ __forceinline__ void mask_rows(int t, int left, Half& h) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * (int)((threadIdx.x & 63) >> 4) + 4 * t + i >= left) h.rc[0][i] = h.rc[1][i] = INFINITY;
  }

  // Vector work on element e = (column, row), in parts of some 12 cycles: a weight,
  __device__ __forceinline__ void weight(Half& h, int m, int e) {
    const int k = e >> 2, i = e & 3;
    h.s[m][k][i] = fast_exp2(fmaf(h.s[m][k][i], c, -h.rc[m][i]));
  }
  // PREV: there is an older tile, `cur`; NEXT: a newer one, t = 0 of it to `nxt`; MORE: and one after that, which is waited for.
  template <bool PREV, bool NEXT, bool MORE>
  __device__ __forceinline__ void body(Packed& cur, Packed& nxt, int newer, int left) {
    bf16x8_t fr[32];
    // All else of an element, in two parts (x: its results, y: those of the row before it).
    float xa, x1, x2, ya, y1, y2;
    auto rest_a = [&](Half& h, int e) {
      const int k = e >> 2, i = e & 3;
      xa = fmaf(-lam, h.s[1][k][i], h.s[0][k][i]);
      x1 = h.s[0][k][i] * (h.dp[k][i] - h.rc[2][i]);
      x2 = h.rc[3][i] - h.dp[k][i];
    };
    auto rest_b = [&](Half& h, int t, int e, Packed& p) {
      const int k = e >> 2, i = e & 3;
      x2 *= h.s[1][k][i];
      if (i & 1) {   // to nearest even: operands of the matrix products
        p.a[k][2 * t + (i >> 1)] = pack_bf16x2(ya, xa);
        p.d1[k][2 * t + (i >> 1)] = pack_bf16x2(y1, x1);
        p.d2[k][2 * t + (i >> 1)] = pack_bf16x2(y2, x2);
      } else {
        ya = xa;
        y1 = x1;
        y2 = x2;
      }
    };
    auto load = [&](int f) {   // in the order of use
      if (!PREV && f >= 8 && f < 24) f += 16;
      if (f < 8) fr[f] = read_nat<32>(nat + (f >> 2) * 4 * Tiles::kTile, 0, f & 3);
      else if (f < 24) fr[f] = read_tr<32>(tr, (f & 1 ? 0 : 4 * Tiles::kTile), (f - 8) >> 1);
      else if (f < 32) fr[f] = NEXT ? read_nat<32>(nat + ((f - 24) >> 2) * 4 * Tiles::kTile, 1, f & 3) : fr[f - 1];
    };
    auto products = [&](int f, Half& h, auto&& vec) {   // the three of a row fragment, and vector work behind each
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const int kb = f & 3;
        floatx4_t& d = f & 4 ? h.dp[k] : h.s[kb >> 1][k];
        d = mfma16(fr[f], f & 4 ? vf[k][kb] : kf[k][kb], kb == 0 || (!(f & 4) && kb == 2) ? floatx4_t{0.f, 0.f, 0.f, 0.f} : d);
        vec(3 * (f & 7) + k);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if constexpr (NEXT) {
#pragma unroll
      for (int f = 0; f < kWin; ++f) fr[f] = ahead[f];
#pragma unroll
      for (int f = 0; f < 8; ++f) {
        load(f + kWin);
        if (f == 4) load_rows(0, h0);
        products(f, h0, [&](int slot) {
          if constexpr (PREV) {
            if (slot & 1) rest_b(h1, 1, slot >> 1, cur);
            else rest_a(h1, slot >> 1);
          }
        });
      }
      if constexpr (!MORE) mask_rows(0, left, h0);
    } else {
      load(8);
      load(9);
#pragma unroll
      for (int e = 0; e < 4 * NC; ++e) {
        rest_a(h1, e);
        rest_b(h1, 1, e, cur);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    auto first_half = [&](int slot) {
      const int e = slot >> 2;
      if ((slot & 3) == 0) weight(h0, 0, e);
      if ((slot & 3) == 1) weight(h0, 1, e);
      if ((slot & 3) == 2) rest_a(h0, e);
      if ((slot & 3) == 3) rest_b(h0, 0, e, nxt);
    };
    if constexpr (PREV) {
#pragma unroll
      for (int f = 8; f < 24; ++f) {
        if (NEXT || f < 22) load(f + kWin);
        if (NEXT && f == 20) load_rows(1, h1);
        const int dt = (f - 8) >> 1;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          if (f & 1) dk[dt][k] = mfma16(fr[f], __builtin_bit_cast(bf16x8_t, dt < 4 ? cur.d1[k] : cur.d2[k]), dk[dt][k]);
          else dv[dt][k] = mfma16(fr[f], __builtin_bit_cast(bf16x8_t, cur.a[k]), dv[dt][k]);
          if constexpr (NEXT) first_half(3 * (f - 8) + k);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
#pragma unroll
      for (int slot = 0; slot < 48; ++slot) {
        first_half(slot);
        __builtin_amdgcn_sched_barrier(0);
      }
      load_rows(1, h1);
    }
    if constexpr (NEXT) {
      if constexpr (!MORE) mask_rows(1, left, h1);
      const unsigned own = nat;
#pragma unroll
      for (int f = 24; f < 32; ++f) {
        if (f < 30) {
          load(PREV ? f + kWin : f - 16 + kWin);
        } else if constexpr (MORE) {
          if (f == 30) {
            tiles.ready(newer + 1);
            nat = in_register(tiles.n_[0] + tiles.off);
          }
          ahead[f - 30] = read_nat<32>(nat, 0, f - 30);
        }
        products(f, h1, [&](int slot) {
          if (slot >= 6 && slot < 18) weight(h1, 0, slot - 6);
          if (slot >= 12) weight(h1, 1, slot - 12);
        });
      }
      // the newer tile is the older one from here on
      const unsigned by = own - tiles.n_[0];
#pragma unroll
      for (int p = 0; p < 2; ++p) tr[p] = in_register(tiles.t_[0][p] + by);
    }
  }

  __device__ __forceinline__ void sweep(int n) {
    const int steps = (n + 31) >> 5;
    Packed p0, p1;
    nat = tiles.n_[0] + tiles.off;
#pragma unroll
    for (int f = 0; f < kWin; ++f) ahead[f] = read_nat<32>(nat, 0, f);
    if (steps > 1) body<false, true, true>(p1, p0, 0, 32);
    else body<false, true, false>(p1, p0, 0, n);
    int s = 0;
    for (; s + 3 < steps; s += 2) {
      body<true, true, true>(p0, p1, s + 1, 32);
      body<true, true, true>(p1, p0, s + 2, 32);
    }
    if (s + 2 < steps) {
      body<true, true, true>(p0, p1, s + 1, 32);
      p0 = p1;
    }
    if (steps > 1) {
      body<true, true, false>(p0, p1, steps - 1, n - 32 * (steps - 1));
      p0 = p1;
    }
    body<true, false, false>(p0, p1, 0, 0);
  }
};

}  // namespace moga
