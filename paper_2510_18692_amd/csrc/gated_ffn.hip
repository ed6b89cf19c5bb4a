// Gated feed-forward, forward and backward.
//
//   [a, u] = x W_in^T,  h = act(a) u,  y = h W_out^T
//   dh = d_y W_out,  da = dh u act'(a),  du = dh act(a),  d_x = [da, du] W_in,  d_W_in = [da, du]^T x,  d_W_out = d_y^T h
//
// Six matrix products, 6 N C F operations forward and 12 N C F backward, the activation and its derivative in the epilogues of the two that make h and dh:
// [a, u] leaves a block's registers once, dh never.  From some hundred tokens on bound by the products (product_kernel), with few tokens by the
// weights' bytes (few_kernel).  h comes from the unrounded a and u, da and du from a and u as the forward kept them (finer()) and the unrounded dh;
// the three are rounded to the inputs' type once, as operands of the next product.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "matmul_tiles.h"

namespace moga {
namespace {

constexpr int kFfnMaxC = 65536, kFfnMaxF = 262144;

// ---- the activation ----
template <typename T> __device__ __forceinline__ float exp_neg(float v);   // e^-v
template <> __device__ __forceinline__ float exp_neg<unsigned short>(float v) { return fast_exp2(v * -1.4426950408889634f); }
template <> __device__ __forceinline__ float exp_neg<float>(float v) { return expf(-v); }
template <typename T> __device__ __forceinline__ float inverse(float v);
template <> __device__ __forceinline__ float inverse<unsigned short>(float v) { return __builtin_amdgcn_rcpf(v); }
template <> __device__ __forceinline__ float inverse<float>(float v) { return 1.f / v; }

// Phi(a), the normal distribution, and e^(-a^2 / 2).  bf16: Abramowitz and Stegun 7.1.26, erfc z = (a1 t + .. + a5 t^5) e^(-z^2) with
// t = 1 / (1 + 0.3275911 z), off by 1.5e-7 at most: 12 instructions on an exponential that the derivative needs anyway.  Relative to Phi that is 5e-4 at
// a = -4, 1.6e-3 at -5, 3.6e-3 at -6 (there gelu is 6e-9) and 2e-2 at -10; half a step of bf16 is 3.9e-3.
// fp32: by erfc, since 1 + erf has nothing left of Phi in its lower tail (2.7e-4 off at a = -4, 4 % at -5, 0 from -6 on).
template <typename T> __device__ __forceinline__ float normal(float a, float& e);
template <> __device__ __forceinline__ float normal<unsigned short>(float a, float& e) {
  e = exp_neg<unsigned short>(0.5f * a * a);
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(a), 0.3275911f * 0.70710678118654752f, 1.f));
  const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, -0.5f * 1.453152027f), 0.5f * 1.421413741f), -0.5f * 0.284496736f),
                           0.5f * 0.254829592f) * e;
  return a < 0.f ? q : 1.f - q;
}
template <> __device__ __forceinline__ float normal<float>(float a, float& e) {
  e = expf(-0.5f * a * a);
  return 0.5f * erfcf(a * -0.70710678118654752f);
}

// act(a) and act'(a).  tanh's form is a sigmoid: (1 + tanh v) / 2 = 1 / (1 + e^-2v).
template <typename T, int ACT>
__device__ __forceinline__ void activate(float a, float& f, float& slope) {
  if constexpr (ACT == MOGA_ACT_SILU) {
    const float p = inverse<T>(1.f + exp_neg<T>(a));
    f = a * p;
    slope = fmaf(f, 1.f - p, p);
  } else if constexpr (ACT == MOGA_ACT_GELU) {
    float e;
    const float p = normal<T>(a, e);
    f = a * p;
    slope = fmaf(a * 0.39894228040143268f, e, p);
  } else {
    constexpr float k = 1.5957691216057308f, c = 0.044715f;   // 2 sqrt(2 / pi); beyond |a| = 100 p is 0 or 1, and a^2 may not be infinite
    const float a2 = fminf(a * a, 1e4f), p = inverse<T>(1.f + exp_neg<T>(k * a * fmaf(c, a2, 1.f)));
    f = a * p;
    slope = fmaf(f * (1.f - p), k * fmaf(3.f * c, a2, 1.f), p);
  }
}
// f(activation) as a constant: one branch for all of a block's values
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
  if (act == MOGA_ACT_SILU) f(std::integral_constant<int, MOGA_ACT_SILU>{});
  else if (act == MOGA_ACT_GELU) f(std::integral_constant<int, MOGA_ACT_GELU>{});
  else f(std::integral_constant<int, MOGA_ACT_GELU_TANH>{});
}

// ---- tiles ----
enum Kind { kPlain, kGated, kGatedBwd };

template <typename T>
struct Product {
  const T *a, *b;        // A(m, k), B(n, k)
  int64_t lda, ldb;
  int64_t M;
  int N, act;            // kGated: N = F, b [2 F][ldb]
  int64_t K;
  T* c;                  // [M][N]; kGated: h; kGatedBwd: [da, du], [M][2 N]
  T* c2;                 // kGated: [a, u], [M][2 N], and finer() behind it, or NULL
  const T* saved;        // kGatedBwd: the same
  // blocks below `whole` have a tile each, the `left` tiles behind them are split along k: block whole + split * left + tile
  unsigned tiles_m, tiles_n, whole, left;
  int64_t k_each;        // k of a split
  float* part;           // their sums, [split][left][BM][BN], or NULL for splits of all of k
};

// What a block does.
struct Work {
  bool is_split;
  unsigned tile, behind, split;   // behind: of the blocks behind `whole`
  template <typename T>
  __device__ __forceinline__ explicit Work(const Product<T>& p) {
    is_split = p.part && blockIdx.x >= p.whole;
    behind = is_split ? blockIdx.x - p.whole : 0;
    split = is_split ? behind / p.left : 0;
    tile = is_split ? p.whole + behind - split * p.left : blockIdx.x;
  }
};
// The product that a tile of two products' list belongs to; it shares k and the list with the first.
template <typename T>
__device__ __forceinline__ void select(Product<T>& p, const Product<T>& second, unsigned& tile) {
  const unsigned tiles = p.tiles_m * p.tiles_n;
  if (tile < tiles) return;
  tile -= tiles;
  p.a = second.a;
  p.b = second.b;
  p.lda = second.lda;
  p.ldb = second.ldb;
  p.M = second.M;
  p.N = second.N;
  p.c = second.c;
  p.tiles_m = second.tiles_m;
  p.tiles_n = second.tiles_n;
}

// a and u go to the backward in bf16 with two more bits each, half a byte a pair: the rounded value's distance from the value, in quarters of a step of
// bf16 from -1/4 on.  What the backward makes of them is rounded itself (da, du); from a and u in bf16 alone the gradients of x and W_in are off by
// 1.76 times what a single rounding of the result is (2-norm, 32,760 x 1536 x 4096), with these bits by 1.45.  A zero stays one.
template <typename T>
__device__ __forceinline__ auto finer(T* c2, int64_t M, int64_t N) {
  return (std::conditional_t<std::is_const_v<T>, const unsigned char, unsigned char>*)(c2 + M * 2 * N);
}
__device__ __forceinline__ unsigned finer_bits(float v, unsigned rounded) {   // rounded: v in bf16, as the upper half
  const int d = (int)(__float_as_uint(v) - rounded);
  return (unsigned)max(0, min(3, (d + 0x6000) >> 14));
}
__device__ __forceinline__ float finer_value(unsigned rounded, unsigned bits) {
  const unsigned v = rounded + (bits << 14) - 0x4000u;
  return __uint_as_float((rounded & 0x7f800000u) == 0x7f800000u ? rounded : v);
}
// Neighbouring columns of a and u, rounded: the bits of all of them, a column's u above its a.
template <int COLS>
__device__ __forceinline__ unsigned finer_pack(const float (&a)[COLS], const float (&u)[COLS], const unsigned (&ra)[COLS / 2], const unsigned (&ru)[COLS / 2]) {
  unsigned all = 0;
#pragma unroll
  for (int i = 0; i < COLS; ++i) {
    const unsigned x = i & 1 ? ra[i / 2] & 0xffff0000u : ra[i / 2] << 16, y = i & 1 ? ru[i / 2] & 0xffff0000u : ru[i / 2] << 16;
    all |= (finer_bits(a[i], x) | finer_bits(u[i], y) << 2) << (4 * i);
  }
  return all;
}

__device__ __forceinline__ uintx2_t pack4(floatx4_t v) { return uintx2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

// The columns of a wave's sums in units of two neighbouring tiles: lane group g holds columns 4 g .. of either.  Lanes exchange fours, after which
// each has eight neighbouring columns, from unit_column(g) on.
__device__ __forceinline__ int unit_column(int g) { return (g & 1) * 16 + (g >> 1) * 8; }
__device__ __forceinline__ void exchange(unsigned& p, unsigned& q) {
  const auto x = __builtin_amdgcn_permlane16_swap(p, q, false, false);
  p = x[0], q = x[1];
}
__device__ __forceinline__ uintx4_t unit_packed(floatx4_t p, floatx4_t q) {
  const uintx2_t x = pack4(p), y = pack4(q);
  unsigned v[4] = {x[0], x[1], y[0], y[1]};
  exchange(v[0], v[2]);
  exchange(v[1], v[3]);
  return uintx4_t{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void unit_eight(floatx4_t p, floatx4_t q, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned x = __float_as_uint(p[i]), y = __float_as_uint(q[i]);
    exchange(x, y);
    v[i] = __uint_as_float(x);
    v[4 + i] = __uint_as_float(y);
  }
}

// A unit of a row of C from column col on, rounded once: 16 bytes a lane.
__device__ __forceinline__ void put_unit(unsigned short* row, int col, int g, int64_t N, bool ok, floatx4_t p, floatx4_t q) {
  const uintx4_t v = unit_packed(p, q);
  col += unit_column(g);
  if (ok && col < N) *(uintx4_t*)(row + col) = v;
}
__device__ __forceinline__ void put_unit(float* row, int col, int g, int64_t N, bool ok, floatx4_t p, floatx4_t q) {
  col += 4 * g;
  if (ok && col < N) *(floatx4_t*)(row + col) = p;
  if (ok && col + 16 < N) *(floatx4_t*)(row + col + 16) = q;
}

// a and u of a unit of a row, as a lane needs them for their gradients.
template <typename T> struct Saved;
template <> struct Saved<unsigned short> {
  uintx4_t a, u;
  unsigned bits;
  __device__ __forceinline__ void load(const unsigned short* row, const unsigned char* fine, int64_t F, int col, int g, bool ok) {
    col += unit_column(g);
    a = u = uintx4_t{0, 0, 0, 0};
    bits = 0;
    if (ok && col < F) {
      a = *(const uintx4_t*)(row + col);
      u = *(const uintx4_t*)(row + F + col);
      bits = *(const unsigned*)(fine + col / 2);
    }
  }
  template <int ACT>
  __device__ __forceinline__ void put(unsigned short* row, int64_t F, int col, int g, bool ok, floatx4_t p, floatx4_t q) const {
    float dh[8];
    unit_eight(p, q, dh);
    uintx4_t da4, du4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float da[2], du[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const unsigned at = 8 * i + 4 * k;
        const float av = finer_value(k ? a[i] & 0xffff0000u : a[i] << 16, bits >> at & 3), uv = finer_value(k ? u[i] & 0xffff0000u : u[i] << 16, bits >> (at + 2) & 3);
        float f, slope;
        activate<unsigned short, ACT>(av, f, slope);
        da[k] = dh[2 * i + k] * uv * slope;
        du[k] = dh[2 * i + k] * f;
      }
      da4[i] = pack_bf16x2(da[0], da[1]);
      du4[i] = pack_bf16x2(du[0], du[1]);
    }
    col += unit_column(g);
    if (ok && col < F) {
      *(uintx4_t*)(row + col) = da4;
      *(uintx4_t*)(row + F + col) = du4;
    }
  }
};
template <> struct Saved<float> {
  floatx4_t a[2], u[2];
  __device__ __forceinline__ void load(const float* row, const unsigned char*, int64_t F, int col, int g, bool ok) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int at = col + 16 * t + 4 * g;
      a[t] = u[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      if (ok && at < F) {
        a[t] = *(const floatx4_t*)(row + at);
        u[t] = *(const floatx4_t*)(row + F + at);
      }
    }
  }
  template <int ACT>
  __device__ __forceinline__ void put(float* row, int64_t F, int col, int g, bool ok, floatx4_t p, floatx4_t q) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int at = col + 16 * t + 4 * g;
      const floatx4_t dh = t ? q : p;
      floatx4_t da, du;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f, s;
        activate<float, ACT>(a[t][i], f, s);
        da[i] = dh[i] * u[t][i] * s;
        du[i] = dh[i] * f;
      }
      if (ok && at < F) {
        *(floatx4_t*)(row + at) = da;
        *(floatx4_t*)(row + F + at) = du;
      }
    }
  }
};

// Eight columns of a row: h, and a and u for the backward.
template <int ACT>
__device__ __forceinline__ void put_gated_eight(const Product<unsigned short>& p, int64_t row, int col, const float (&a)[8], const float (&u)[8]) {
  const int64_t N = p.N;
  uintx4_t h;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f0, f1, slope;
    activate<unsigned short, ACT>(a[2 * i], f0, slope);
    activate<unsigned short, ACT>(a[2 * i + 1], f1, slope);
    h[i] = pack_bf16x2(f0 * u[2 * i], f1 * u[2 * i + 1]);
  }
  *(uintx4_t*)(p.c + row * N + col) = h;
  if (p.c2) {
    unsigned ra[4], ru[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ra[i] = pack_bf16x2(a[2 * i], a[2 * i + 1]);
      ru[i] = pack_bf16x2(u[2 * i], u[2 * i + 1]);
    }
    *(uintx4_t*)(p.c2 + row * 2 * N + col) = uintx4_t{ra[0], ra[1], ra[2], ra[3]};
    *(uintx4_t*)(p.c2 + row * 2 * N + N + col) = uintx4_t{ru[0], ru[1], ru[2], ru[3]};
    *(unsigned*)(finer(p.c2, p.M, N) + row * N / 2 + col / 2) = finer_pack<8>(a, u, ra, ru);
  }
}

// A row's h, and its a and u for the backward, of 32 columns from col on: a's sums in a0 and a1, u's in u0 and u1.
template <int ACT>
__device__ __forceinline__ void put_gated(const Product<unsigned short>& p, int64_t row, int col, int g, bool ok, floatx4_t a0, floatx4_t a1, floatx4_t u0,
                                          floatx4_t u1) {
  float a[8], u[8];
  unit_eight(a0, a1, a);
  unit_eight(u0, u1, u);
  col += unit_column(g);
  if (ok && col < p.N) put_gated_eight<ACT>(p, row, col, a, u);
}
template <int ACT>
__device__ __forceinline__ void put_gated(const Product<float>& p, int64_t row, int col, int g, bool ok, floatx4_t a0, floatx4_t a1, floatx4_t u0,
                                          floatx4_t u1) {
  const int64_t N = p.N;
  floatx4_t h[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f, slope;
      activate<float, ACT>(t ? a1[i] : a0[i], f, slope);
      h[t][i] = f * (t ? u1[i] : u0[i]);
    }
  put_unit(p.c + row * N, col, g, N, ok, h[0], h[1]);
  if (p.c2) {
    put_unit(p.c2 + row * 2 * N, col, g, N, ok, a0, a1);
    put_unit(p.c2 + row * 2 * N + N, col, g, N, ok, u0, u1);
  }
}

// One tile of a product: WM x WN waves, TM x TN tiles of 16 x 16 each.
//
// Blocks of 256 x 256 (a CU each) read 2 bytes of operands from the caches for 256 operations, twice the reuse of 128 x 128 (two to a CU).  A step's two halves
// of k alternate: the operands of a half are read from LDS while the products of the other run, and the loads of the step after next go out one with
// each row of tiles; a step has one barrier.  A row of tiles goes out in whole 16 bytes a lane (permlane exchange), without a trip through LDS.
//
// bf16, 32,760 tokens, us and TFLOP/s by kernel (the forward without a backward; a library's square product of 16,384 reaches 1,530 on the same card):
//                                      C 1536, F 4096     C 5120, F 13696
//   in  (kGated, rows x rows)          772   1,070        7,212   1,270
//   out (kPlain, rows x rows)          342   1,210        3,318   1,380
//   dh  (kGatedBwd, rows x columns)    560     740        4,059   1,130
//   dx  (kPlain, rows x columns)       618   1,330        6,546   1,400
//   dW_in, dW_out (columns x columns)  963 + 12 to join  1,280   9,964 + 35  1,380
// The long products are bound by power: the matrix cores are busy 0.71 to 0.75 of the cycles at 1.75 to 1.85 GHz of 2.4.  Fed from no loads at all the loop
// makes 1,650 to 1,730, from loads of the same lines over and over 1,430 to 1,500: the rest is what bringing 64 KB a step from the caches costs in time
// and in clock.  LDS has no bank conflicts and is busy 0.28 of the cycles.  With C = 1536 a tile's 24 steps (35 us) are followed by its epilogue,
// beside which its CU has no products: dh takes 358 us without its 544 KB a block of a, u, da and du, 434 with the loads alone, 466 with the stores alone.
// Starting half of the CUs half a tile later puts that traffic beside the others' products and gains nothing.
// Fp32, 8,192 x 4096 x 4096, blocks of 128: 143 TFLOP/s of rows x rows, 129 to 132 with columns (4-byte reads), of a library's 153.
template <typename T, Kind KIND, bool A_KFIRST, bool B_KFIRST, int WM, int WN, int TM, int TN>
__device__ __forceinline__ void product_tile(const Product<T>& p, const Work& work) {
  constexpr int THREADS = 64 * WM * WN, BM = 16 * WM * TM, BN = 16 * WN * TN;
  using OpA = Operand<T, A_KFIRST, BM, THREADS, TM>;
  using OpB = Operand<T, B_KFIRST, BN, THREADS, TN>;
  constexpr int BK = OpA::BK;
  constexpr unsigned kStage = OpA::kBytes + OpB::kBytes;
  __shared__ __attribute__((aligned(1024))) unsigned char s_mem[2 * kStage];
  const unsigned lds = lds_addr_uniform(s_mem);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;

  unsigned bm, bn;
  tile_of(work.tile, p.tiles_m, p.tiles_n, bm, bn);

  const int64_t m0 = (int64_t)bm * BM, k0 = work.split * p.k_each;
  const int n0 = bn * (KIND == kGated ? BN / 2 : BN), k_count = (int)(work.is_split ? min(p.k_each, p.K - k0) : p.K);
  OpA oa;
  OpB ob;
  oa.init(p.a, p.lda, m0, p.M, k0, k_count, wm * TM, lds);
  if constexpr (KIND == kGated) ob.init_paired(p.b + k0, p.ldb, n0, p.N, k_count, wn * TN, lds + OpA::kBytes);
  else ob.init(p.b, p.ldb, n0, p.N, k0, k_count, wn * TN, lds + OpA::kBytes);

  // the i-th of the thread's loads of a step; past the last step they are zeros
  constexpr int LOADS = OpA::L + OpB::L;
  auto load = [&](int i) {
    if (i < OpA::L) oa.stage(i);
    else ob.template stage<KIND == kGated>(i - OpA::L);
  };
  auto advance = [&](int other) {
    oa.advance(other);
    ob.template advance<KIND == kGated>(other);
  };

  floatx4_t acc[TM][TN];
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int n = 0; n < TN; ++n) acc[m][n] = floatx4_t{0.f, 0.f, 0.f, 0.f};

  // While the products of half a step run, the operands of the next half are read, each into the registers of the one just used.  Behind the first
  // products of the second half one barrier: all of the step's buffer is in registers, so that the loads of the step after next go out into it, and
  // the next step's has landed.
  Frag<T> fa[TM], fb[2][TN];
  auto half = [&](auto which) {
    constexpr int H = which.value, PER = (LOADS + TM - 1) / TM, FB = (TN + TM - 1) / TM;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
      for (int n = 0; n < TN; ++n) mfma_frag(acc[m][n], fb[H][n], fa[m]);
      if (H == 1 && m == 0) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      if (H == 1)
#pragma unroll
        for (int i = m * PER; i < (m + 1) * PER && i < LOADS; ++i) load(i);
      fa[m] = oa.get(m, 1 - H);
#pragma unroll
      for (int n = m * FB; n < (m + 1) * FB && n < TN; ++n) fb[1 - H][n] = ob.get(n, 1 - H);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int other = kStage;
#pragma unroll
  for (int i = 0; i < LOADS; ++i) load(i);
  advance(other);
#pragma unroll
  for (int i = 0; i < LOADS; ++i) load(i);
  advance(-other);
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(LOADS));
  block_barrier();
#pragma unroll
  for (int n = 0; n < TN; ++n) fb[0][n] = ob.get(n, 0);
#pragma unroll
  for (int m = 0; m < TM; ++m) fa[m] = oa.get(m, 0);
  if constexpr (!A_KFIRST) oa.turn(0, other);
  if constexpr (!B_KFIRST) ob.turn(0, other);
  for (int left = (k_count - 1) / BK; left >= 0; --left) {
    half(std::integral_constant<int, 0>{});
    if constexpr (A_KFIRST) oa.turn(0, other);
    if constexpr (B_KFIRST) ob.turn(0, other);
    half(std::integral_constant<int, 1>{});
    oa.turn(1, other);
    ob.turn(1, other);
    advance(other);
    other = -other;
    if constexpr (!A_KFIRST) oa.turn(0, other);
    if constexpr (!B_KFIRST) ob.turn(0, other);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way into this block's LDS when it ends

  // lane: row r of a tile, columns 4 g .. 4 g + 3
  constexpr int UNITS = TN / 2;
  const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int64_t N = p.N;
  const int col0 = n0 + wn * TN * 16;
  if (work.is_split) {
    float* out = p.part + (size_t)work.behind * BM * BN + wn * TN * 16;
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
      for (int n = 0; n < TN; ++n) *(floatx4_t*)(out + ((wm * TM + m) * 16 + r) * BN + 16 * n + 4 * g) = acc[m][n];
    return;
  }
  // the saved rows of AHEAD rows of tiles are on their way: of one 550 us (32,760 x 1536 x 4096), of two 541, of three, which do
  // not fit the registers, 622
  constexpr int AHEAD = KIND == kGatedBwd ? 2 : 1, FETCHED = KIND == kGatedBwd ? UNITS : 1;
  Saved<T> saved[AHEAD][FETCHED];
  auto fetch_saved = [&](int m) {
    const int64_t row = m0 + (wm * TM + m) * 16 + r;
#pragma unroll
    for (int u = 0; u < FETCHED; ++u) saved[m % AHEAD][u].load(p.saved + row * 2 * N, finer(p.saved, p.M, N) + row * N / 2, N, col0 + 32 * u, g, row < p.M);
  };
  auto rows = [&](auto act) {
    constexpr int ACT = act.value;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      const int64_t row = m0 + (wm * TM + m) * 16 + r;
      const bool ok = row < p.M;
      __builtin_amdgcn_sched_barrier(0);   // a row of tiles at a time: all of them do not fit the registers
      if constexpr (KIND == kPlain) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) put_unit(p.c + row * N, col0 + 32 * u, g, N, ok, acc[m][2 * u], acc[m][2 * u + 1]);
      } else if constexpr (KIND == kGated) {
        static_assert(UNITS == 2);   // of 64 columns the first unit is a's, the second u's
        const int col = n0 + wn * TN * 8;
        put_gated<ACT>(p, row, col, g, ok, acc[m][0], acc[m][1], acc[m][2], acc[m][3]);
      } else {
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
          saved[m % AHEAD][u].template put<ACT>(p.c + row * 2 * N, N, col0 + 32 * u, g, ok, acc[m][2 * u], acc[m][2 * u + 1]);
        if (m + AHEAD < TM) fetch_saved(m + AHEAD);
      }
    }
  };
  if constexpr (KIND == kGatedBwd)
#pragma unroll
    for (int m = 0; m < AHEAD && m < TM; ++m) fetch_saved(m);
  if constexpr (KIND == kPlain) rows(std::integral_constant<int, 0>{});
  else with_activation(p.act, rows);
}
template <typename T, Kind KIND, bool A_KFIRST, bool B_KFIRST, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN, TM == 2 ? 3 : 2) void product_kernel(const Product<T> p) {
  product_tile<T, KIND, A_KFIRST, B_KFIRST, WM, WN, TM, TN>(p, Work(p));
}
// Two products of the same k in one list of tiles: fewer of them are behind the last whole round.
template <typename T, bool A_KFIRST, bool B_KFIRST, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN, TM == 2 ? 3 : 2) void product_pair_kernel(Product<T> p, const Product<T> second) {
  Work work(p);
  select(p, second, work.tile);
  product_tile<T, kPlain, A_KFIRST, B_KFIRST, WM, WN, TM, TN>(p, work);
}

// Tiles that were split along k: the sums of their splits, in order (results repeat bit by bit), and what a block does with its sums.  A thread has eight
// columns of a row (kGated: of a, and the same eight of u); blockIdx.x is the tile, blockIdx.y a run of its rows.  Bound by the partial sums' bytes, which
// come from the cache behind the L2s where they fit: 148 tiles of 256 x 256 in five splits (194 MB) 35 us, 5.5 TB/s.
template <typename T, Kind KIND, int BM, int BN>
__device__ __forceinline__ void join_tile(const Product<T>& p, unsigned tile, int splits) {
  constexpr int COLS = KIND == kGated ? BN / 2 : BN, SETS = KIND == kGated ? 2 : 1, PER = COLS / 8;
  unsigned bm, bn;
  tile_of(tile, p.tiles_m, p.tiles_n, bm, bn);
  const int at = blockIdx.y * 256 + threadIdx.x, r = at / PER, c = at % PER * 8;
  const int64_t row = (int64_t)bm * BM + r, N = p.N;
  const int col = bn * COLS + c;
  if (row >= p.M || col >= N) return;
  floatx4_t v[SETS][2];
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    // of each 64 staged columns 32 are a's, 32 u's
    const float* in = p.part + ((size_t)blockIdx.x * BM + r) * BN + (KIND == kGated ? (c >> 5) * 64 + s * 32 + (c & 31) : c);
    v[s][0] = v[s][1] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
      v[s][0] += *(const floatx4_t*)(in + (size_t)k * p.left * BM * BN);
      v[s][1] += *(const floatx4_t*)(in + (size_t)k * p.left * BM * BN + 4);
    }
  }
  // fp32: N is a multiple of 4
  auto put = [&](T* to, floatx4_t x, floatx4_t y) {
    if constexpr (sizeof(T) == 4) {
      *(floatx4_t*)to = x;
      if (col + 4 < N) *(floatx4_t*)(to + 4) = y;
    } else {
      const uintx2_t a = pack4(x), b = pack4(y);
      *(uintx4_t*)to = uintx4_t{a[0], a[1], b[0], b[1]};
    }
  };
  auto take = [&](const T* from, floatx4_t (&x)[2]) {
    if constexpr (sizeof(T) == 4) {
      x[0] = *(const floatx4_t*)from;
      x[1] = col + 4 < N ? *(const floatx4_t*)(from + 4) : floatx4_t{0.f, 0.f, 0.f, 0.f};
    } else {
      const uintx4_t b = *(const uintx4_t*)from;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) x[t][2 * i] = bf16_lo_to_f32(b[2 * t + i]), x[t][2 * i + 1] = bf16_hi_to_f32(b[2 * t + i]);
    }
  };
  if constexpr (KIND == kPlain) {
    put(p.c + row * N + col, v[0][0], v[0][1]);
  } else {
    with_activation(p.act, [&](auto act) {
      if constexpr (KIND == kGated && sizeof(T) == 2) {
        float a[8], u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = v[0][i / 4][i % 4], u[i] = v[1][i / 4][i % 4];
        put_gated_eight<act.value>(p, row, col, a, u);
      } else if constexpr (KIND == kGated) {
        floatx4_t h[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float f, slope;
            activate<T, act.value>(v[0][t][i], f, slope);
            h[t][i] = f * v[1][t][i];
          }
        put(p.c + row * N + col, h[0], h[1]);
        if (p.c2) {
          put(p.c2 + row * 2 * N + col, v[0][0], v[0][1]);
          put(p.c2 + row * 2 * N + N + col, v[1][0], v[1][1]);
        }
      } else {
        floatx4_t a[2], u[2], da[2], du[2];
        const T* at = p.saved + row * 2 * N + col;
        take(at, a);
        take(at + N, u);
        if constexpr (sizeof(T) == 2) {
          const unsigned bits = *(const unsigned*)(finer(p.saved, p.M, N) + row * N / 2 + col / 2);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            a[i / 4][i % 4] = finer_value(__float_as_uint(a[i / 4][i % 4]), bits >> 4 * i & 3);
            u[i / 4][i % 4] = finer_value(__float_as_uint(u[i / 4][i % 4]), bits >> (4 * i + 2) & 3);
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float f, slope;
            activate<T, act.value>(a[t][i], f, slope);
            da[t][i] = v[0][t][i] * u[t][i] * slope;
            du[t][i] = v[0][t][i] * f;
          }
        put(p.c + row * 2 * N + col, da[0], da[1]);
        put(p.c + row * 2 * N + N + col, du[0], du[1]);
      }
    });
  }
}
template <typename T, Kind KIND, int BM, int BN>
__global__ __launch_bounds__(256) void join_kernel(const Product<T> p, int splits) {
  join_tile<T, KIND, BM, BN>(p, p.whole + blockIdx.x, splits);
}
template <typename T, int BM, int BN>
__global__ __launch_bounds__(256) void join_pair_kernel(Product<T> p, const Product<T> second, int splits) {
  unsigned tile = p.whole + blockIdx.x;
  select(p, second, tile);
  join_tile<T, kPlain, BM, BN>(p, tile, splits);
}

// ---- few tokens ----
// A block owns 16 columns of C (GATED: 16 of a and the same 16 of u) for up to 16 TT tokens.  Its waves take turns of 128 bytes of k, so that a weight
// is read once, a line at a time, and their sums meet in LDS.  Loads past k, F or the last token give zeros (buffer bounds).  The products of 16 tokens cost
// a matrix instruction what one token's cost it, so there is no form for a single one.
// Bound by HBM: 1 token, C 5120, F 13696, bf16: 53 us for W_in's 281 MB, 25 for W_out's 140 and 5 for the join (5.3 and 5.6 TB/s of weights, some of them
// from the cache behind the L2s where passes follow each other).  24 tokens, 1536 x 4096: 8.2, 5.8 and 2.2 us, launches and their chain of loads.
// The second product without its split and join, in blocks of 16 waves: 11.2 us instead of 8.0, of 8 columns a block 10.0; 1 token 33 instead of 24.
template <typename T, bool GATED, int TT, int WAVES, int U>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(const Product<T> p) {
  constexpr int ES = sizeof(T), SETS = GATED ? 2 : 1;
  __shared__ floatx4_t s_sum[WAVES][SETS * TT][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, r = l & 15, g = l >> 4;
  const int n0 = blockIdx.x * 16, N = p.N;
  const int row_bytes = (int)(p.ldb * ES);
  // this block's bytes of a row
  const int first = (int)(blockIdx.y * p.k_each * ES), end = min(row_bytes, first + (int)(p.k_each * ES));
  auto rsrc = [](const T* base) { return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)kBufferBytes, 0x00020000); };
  const auto ra = rsrc(p.a);
  const auto rb = rsrc(p.b + (int64_t)n0 * p.ldb), rb2 = rsrc(p.b + ((int64_t)N + n0) * p.ldb);
  const unsigned vb = n0 + r < N ? r * row_bytes + g * 16 : kPastBuffer;
  unsigned va[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) va[t] = 16 * t + r < p.M ? (16 * t + r) * row_bytes + g * 16 : kPastBuffer;
  floatx4_t acc[SETS][TT];
#pragma unroll
  for (int s = 0; s < SETS; ++s)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[s][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  // two sets of U lines in turn: one on its way while the products of the other run
  Frag<T> fb[2][U][2][SETS], fa[2][U][2][TT];
  auto fetch = [&](auto which, int k) {
    constexpr int H = which.value;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = k + u * WAVES * 128 + h * 64;
        const bool in = at + g * 16 < end;
        const unsigned b = in ? vb : kPastBuffer;
        auto get = [&](auto& f, auto rs, unsigned v) { f.v = __builtin_bit_cast(decltype(f.v), __builtin_amdgcn_raw_buffer_load_b128(rs, v, at, 0)); };
        get(fb[H][u][h][0], rb, b);
        if constexpr (GATED) get(fb[H][u][h][1], rb2, b);
#pragma unroll
        for (int t = 0; t < TT; ++t) get(fa[H][u][h][t], ra, in ? va[t] : kPastBuffer);
      }
  };
  auto multiply = [&](auto which) {
    constexpr int H = which.value;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
          for (int s = 0; s < SETS; ++s) mfma_frag(acc[s][t], fb[H][u][h][s], fa[H][u][h][t]);
  };
  constexpr int STEP = WAVES * 128 * U;
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  int k = first + wave * 128;
  if (k < end) fetch(even, k);
  for (; k < end; k += 2 * STEP) {
    if (k + STEP < end) fetch(odd, k + STEP);
    multiply(even);
    if (k + STEP >= end) break;
    if (k + 2 * STEP < end) fetch(even, k + 2 * STEP);
    multiply(odd);
  }
#pragma unroll
  for (int s = 0; s < SETS; ++s)
#pragma unroll
    for (int t = 0; t < TT; ++t) s_sum[wave][s * TT + t][l] = acc[s][t];
  __syncthreads();
  for (int t = wave; t < TT; t += WAVES) {
    const int64_t row = 16 * t + r;
    const int col = n0 + 4 * g;
    floatx4_t v[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      v[s] = s_sum[0][s * TT + t][l];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v[s] += s_sum[w][s * TT + t][l];
    }
    if (row >= p.M || col >= N) continue;
    if (!GATED && p.part) {
      *(floatx4_t*)(p.part + ((int64_t)blockIdx.y * p.M + row) * N + col) = v[0];
      continue;
    }
    auto put = [&](T* at, floatx4_t x) {
      if constexpr (ES == 4) *(floatx4_t*)at = x;
      else *(uintx2_t*)at = pack4(x);
    };
    if constexpr (GATED) {
      floatx4_t h;
      with_activation(p.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f, slope;
          activate<T, act.value>(v[0][i], f, slope);
          h[i] = f * v[1][i];
        }
      });
      put(p.c + row * N + col, h);
      if (p.c2) {
        put(p.c2 + row * 2 * N + col, v[0]);
        put(p.c2 + row * 2 * N + N + col, v[1]);
        if constexpr (ES == 2) {
          const uintx2_t x = pack4(v[0]), y = pack4(v[1]);
          const float a[4] = {v[0][0], v[0][1], v[0][2], v[0][3]}, u[4] = {v[1][0], v[1][1], v[1][2], v[1][3]};
          const unsigned ra[2] = {x[0], x[1]}, ru[2] = {y[0], y[1]};
          *(unsigned short*)(finer(p.c2, p.M, N) + row * N / 2 + col / 2) = (unsigned short)finer_pack<4>(a, u, ra, ru);
        }
      }
    } else {
      put(p.c + row * N + col, v[0]);
    }
  }
}

// Sums of the splits of few tokens' rows, in order, rounded once.  Bound by its launch and one chain of loads (2.2 to 4.7 us).
template <typename T>
__global__ __launch_bounds__(64) void few_join_kernel(const float* __restrict__ part, int splits, int64_t n, T* __restrict__ c) {
  const int64_t i = ((int64_t)blockIdx.x * 64 + threadIdx.x) * 4;
  if (i >= n) return;
  floatx4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = 0; k < splits; ++k) s += *(const floatx4_t*)(part + k * n + i);
  if constexpr (sizeof(T) == 4) *(floatx4_t*)(c + i) = s;
  else *(uintx2_t*)(c + i) = pack4(s);
}

// ---- host ----
constexpr int kFewTokens = 64, kFewBlocks = 1280;

// Few tokens go by the weights' rows: 16 at least, more while what their blocks read of x (N C F / 8 values, some 9 TB/s from the caches) takes less
// than what tiles cost beside the weights, 10 us and a tenth of their time.  bf16, us by rows and by tiles: 64 x 1536 x 4096 23 and 26, 16 x 5120 x
// 13696 103 and 112, 17 tokens 123 and 112; fp32, where tiles of 128 are bound by their products: 64 x 1536 x 4096 41 and 67.
bool few_tokens(int64_t N, int C, int F, int dtype) {
  if (N <= 16 || dtype == MOGA_F32) return N <= kFewTokens;
  const double weights = 3. * C * F * 2 / 4.7e6;
  return N <= kFewTokens && (double)N * C * F / 8 * 2 / 9e6 <= 10 + 0.1 * weights;
}

// How a product is cut: blocks of 256 x 256, 128 x 128 or 64 x 128, whole rounds of them, and the tiles behind those in `splits` runs of k_each along k.
// The cheapest by a model of measured costs.  us of blocks of 256 x 256, 128 x 128 and 64 x 128, bf16: in of 1,563 x 1536 x 4104 45, 54, 63; dh 52, 36, 50;
// dh of 32,760 tokens with k 512 (F 2048) 185, 215, 202 and k 1,536 (F 4096) 560, 643, 725; fp32, in of 2,050 x 512 x 1368 -, 72, 57.  dW_in of 32,760 x 1536
// x 4096 alone, 192 tiles of 256 x 256: in four splits 637 + 37, whole 706.
struct TileShape {
  int bm, bn, resident;       // rows and columns; blocks on the chip at a time
  int threads() const { return bn * 2; }
  // microseconds: a step of bf16 and of fp32 with all of them running, a block's start and end, what writing a split's sums adds to it
  double step, step32, ends, sums;
};
constexpr TileShape kTiles[] = {{256, 256, 256, 1.45, 0, 12, 6}, {128, 128, 512, 1.0, 4.1, 7, 3}, {64, 128, 768, 0.9, 3.2, 6, 2}};
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
struct Cut {
  int shape, splits;
  int64_t k_each;
  unsigned whole, left;
  double cost;
  bool fits() const { return splits > 0; }   // a launch of fewer than 2^32 threads
  size_t part_bytes() const { return splits > 1 ? (size_t)splits * left * kTiles[shape].bm * kTiles[shape].bn * sizeof(float) : 0; }
};
struct Size {
  int64_t M, N;
  unsigned tiles_m(const TileShape& t) const { return (unsigned)ceil_div(M, t.bm); }
  unsigned tiles_n(const TileShape& t, Kind kind) const { return (unsigned)ceil_div(N, kind == kGated ? t.bn / 2 : t.bn); }
};

constexpr int kMostSplits = 32;
double step_of(const TileShape& t, int dtype) { return dtype == MOGA_F32 ? t.step32 : t.step; }
int steps_of(int64_t K, int dtype) { return (int)ceil_div(K, dtype == MOGA_F32 ? 32 : 64); }
int first_shape(int dtype) { return dtype == MOGA_F32 ? 1 : 0; }

// Splits of the tiles behind the last whole round.
struct Splits {
  int s;
  double cost;
};
Splits splits_of(const TileShape& t, int64_t left, int64_t steps, double step) {
  Splits best{};
  const double mb = t.bm * t.bn * 4e-6;   // a tile's sums in MB
  for (int s = 1; s <= kMostSplits; ++s) {
    const int64_t each = ceil_div(steps, s);
    if (s > 1 && (left == 0 || each < 4 || ceil_div(steps, each) != s)) continue;
    double cost = left ? ceil_div(left * s, t.resident) * (each * step + t.ends) : 0;
    if (s > 1) cost += 5 + ceil_div(left * s, t.resident) * t.sums + left * s * mb * 0.27;
    if (best.s == 0 || cost < best.cost) best = {s, cost};
  }
  return best;
}

// Test hook: tiles of one shape, `round` of them to a round, those behind the last whole round in `splits` where k has as many steps, both weights' gradients in
// one list or not.  In one word, so that a call sees all of it; 0: none.
struct Forced {
  int shape, round, splits, together;
};
std::atomic<long long> g_forced{0};
bool forced(Forced& f) {
  const long long v = g_forced.load();
  f = {(int)(v & 255) - 1, (int)(v >> 24), (int)(v >> 8 & 255), (int)(v >> 16 & 255)};
  return v != 0;
}

// Of one product, or of several of the same k in one list of tiles; of no shape (fits()) where none does.
Cut cut_of(std::initializer_list<Size> sizes, int64_t K, int dtype, Kind kind) {
  const int bk = dtype == MOGA_F32 ? 32 : 64;
  const int64_t steps = steps_of(K, dtype);
  Cut best{};
  Forced f;
  const bool is_forced = forced(f);
  for (int shape = first_shape(dtype); shape < 3; ++shape) {
    if (is_forced && shape != std::max(f.shape, first_shape(dtype))) continue;
    TileShape t = kTiles[shape];
    if (is_forced) t.resident = f.round;
    const double step = step_of(t, dtype);
    int64_t tiles = 0;
    for (const Size& size : sizes) tiles += (int64_t)size.tiles_m(t) * size.tiles_n(t, kind);
    if (!grid_fits(tiles + kMostSplits * t.resident, t.threads())) continue;
    const int64_t whole = tiles / t.resident * t.resident, left = tiles - whole;
    const Splits split = is_forced ? Splits{left ? (int)ceil_div(steps, ceil_div(steps, f.splits)) : 1, 0.} : splits_of(t, left, steps, step);
    const double cost = whole / t.resident * (steps * step + t.ends) + split.cost;
    if (best.splits == 0 || cost < best.cost)
      best = {shape, split.s, split.s > 1 ? ceil_div(steps, split.s) * bk : K, (unsigned)(split.s > 1 ? whole : tiles), (unsigned)(split.s > 1 ? left : 0), cost};
  }
  return best;
}
Cut cut_of(int64_t M, int64_t N, int64_t K, int dtype, Kind kind) { return cut_of({{M, N}}, K, dtype, kind); }

// Bytes of the splits of a product of any number of rows up to M.  Tiles behind the last whole round repeat after `resident` rows of tiles.
size_t most_part_bytes(int64_t M, int64_t N, int64_t K, int dtype, Kind kind) {
  size_t most = 0;
  for (int shape = first_shape(dtype); shape < 3; ++shape) {
    const TileShape& t = kTiles[shape];
    const Size size{M, N};
    for (int64_t m = std::min<int64_t>(size.tiles_m(t), t.resident); m > 0; --m) {
      const int64_t left = m * size.tiles_n(t, kind) % t.resident;
      const int s = splits_of(t, left, steps_of(K, dtype), step_of(t, dtype)).s;
      if (s > 1) most = std::max(most, (size_t)s * left * t.bm * t.bn * sizeof(float));
    }
  }
  return most;
}
// Of products of any k up to K: beyond 1,024 steps as for all splits that there are.
size_t most_part_bytes_k(std::initializer_list<Size> sizes, int64_t K, int dtype) {
  size_t most = 0;
  for (int shape = first_shape(dtype); shape < 3; ++shape) {
    const TileShape& t = kTiles[shape];
    int64_t tiles = 0;
    for (const Size& size : sizes) tiles += (int64_t)size.tiles_m(t) * size.tiles_n(t, kPlain);
    const int64_t left = tiles % t.resident;
    const int steps = steps_of(K, dtype);
    int s = left && steps > 1024 ? kMostSplits : 1;
    for (int k = std::min(steps, 1024); left && k > 0; --k) s = std::max(s, splits_of(t, left, k, step_of(t, dtype)).s);
    if (s > 1) most = std::max(most, (size_t)s * left * t.bm * t.bn * sizeof(float));
  }
  return most;
}

template <typename T>
void apply_cut(Product<T>& p, const Cut& c, Kind kind, void* part) {
  const Size size{p.M, p.N};
  p.tiles_m = size.tiles_m(kTiles[c.shape]);
  p.tiles_n = size.tiles_n(kTiles[c.shape], kind);
  p.whole = c.whole;
  p.left = c.left;
  p.k_each = c.k_each;
  p.part = c.splits > 1 ? (float*)part : nullptr;
}
// f(waves along n, rows of tiles of a wave), as constants
template <typename T, typename F>
void with_tiles(int shape, F&& f) {
  if constexpr (sizeof(T) == 2) {
    if (shape == 0) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
  }
  if (shape == 1) f(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, 2>{}, std::integral_constant<int, 2>{});
}

template <typename T, Kind KIND, bool AK, bool BK>
void launch_product(Product<T> p, int dtype, void* part, hipStream_t st) {
  const Cut c = cut_of(p.M, p.N, p.K, dtype, KIND);
  apply_cut(p, c, KIND, part);
  with_tiles<T>(c.shape, [&](auto wn, auto tm) {
    constexpr int WN = wn.value, TM = tm.value, BM = 32 * TM, BN = 64 * WN;
    product_kernel<T, KIND, AK, BK, 2, WN, TM, 4><<<p.whole + p.left * c.splits, 128 * WN, 0, st>>>(p);
    if (p.left) join_kernel<T, KIND, BM, BN><<<dim3(p.left, BM * BN / (KIND == kGated ? 4096 : 2048)), 256, 0, st>>>(p, c.splits);
  });
}

// Two products of the same k, in one list of tiles where that takes fewer rounds.  Both weights' gradients of 32,760 x 1536 x 4096: 288 tiles, a whole round and
// 32 in eight splits, 963 + 12 us; by themselves 192 in four splits and 96 in five, 1,037 us.  2,050 x 512 x 1368 fp32 105 and 107 us.
template <typename T, bool AK, bool BK>
void launch_two(Product<T> p, Product<T> q, int dtype, void* part, hipStream_t st) {
  const Cut c = cut_of({{p.M, p.N}, {q.M, q.N}}, p.K, dtype, kPlain);
  Forced f;
  if (forced(f) ? !f.together : !c.fits() || c.cost >= cut_of(p.M, p.N, p.K, dtype, kPlain).cost + cut_of(q.M, q.N, q.K, dtype, kPlain).cost) {
    launch_product<T, kPlain, AK, BK>(p, dtype, part, st);
    return launch_product<T, kPlain, AK, BK>(q, dtype, part, st);
  }
  apply_cut(p, c, kPlain, part);
  apply_cut(q, c, kPlain, part);
  with_tiles<T>(c.shape, [&](auto wn, auto tm) {
    constexpr int WN = wn.value, TM = tm.value, BM = 32 * TM, BN = 64 * WN;
    product_pair_kernel<T, AK, BK, 2, WN, TM, 4><<<p.whole + p.left * c.splits, 128 * WN, 0, st>>>(p, q);
    if (p.left) join_pair_kernel<T, BM, BN><<<dim3(p.left, BM * BN / 2048), 256, 0, st>>>(p, q, c.splits);
  });
}

// Few tokens: a block for every 16 columns and, of a plain product with fewer than kFewBlocks of those, every run of k, no shorter than 1 KB.
int64_t few_splits(int N, int64_t K, int dtype) {
  const int64_t blocks = ceil_div(N, 16), bytes = K * elem_size(dtype);
  const int64_t s = std::max<int64_t>(1, std::min({(int64_t)16, kFewBlocks / blocks, bytes / 1024}));
  return ceil_div(bytes, ceil_div(ceil_div(bytes, s), 1024) * 1024);
}
size_t few_part_bytes(int64_t M, int N, int64_t K, int dtype) {
  const int64_t s = few_splits(N, K, dtype);
  return s > 1 ? (size_t)s * M * N * sizeof(float) : 0;
}

template <typename T, bool GATED>
void launch_few(Product<T> p, int dtype, void* part, hipStream_t st) {
  const int64_t splits = GATED ? 1 : few_splits(p.N, p.K, dtype), bytes = p.K * sizeof(T);
  p.k_each = splits > 1 ? ceil_div(ceil_div(bytes, splits), 1024) * 1024 / sizeof(T) : p.K;
  p.part = splits > 1 ? (float*)part : nullptr;
  const dim3 blocks((unsigned)ceil_div(p.N, 16), (unsigned)splits);
  if (p.M <= 16) few_kernel<T, GATED, 1, 4, 2><<<blocks, 256, 0, st>>>(p);
  else if (p.M <= 32) few_kernel<T, GATED, 2, 4, 1><<<blocks, 256, 0, st>>>(p);
  else few_kernel<T, GATED, 4, 4, 1><<<blocks, 256, 0, st>>>(p);
  if (splits > 1) {
    const int64_t n = p.M * p.N;
    few_join_kernel<T><<<(unsigned)ceil_div(n, 256), 64, 0, st>>>(p.part, (int)splits, n, p.c);
  }
}

template <typename T>
Product<T> product(const void* a, int64_t lda, const void* b, int64_t ldb, int64_t M, int N, int64_t K, void* c) {
  Product<T> p{};
  p.a = (const T*)a;
  p.b = (const T*)b;
  p.lda = lda;
  p.ldb = ldb;
  p.M = M;
  p.N = N;
  p.K = K;
  p.c = (T*)c;
  return p;
}

template <typename T>
void ffn_fwd(const void* x, const void* w_in, const void* w_out, int dtype, int64_t N, int C, int F, int act, void* h, void* au, void* y, void* ws,
             hipStream_t st) {
  Product<T> in = product<T>(x, C, w_in, C, N, F, C, h);
  in.c2 = (T*)au;
  in.act = act;
  const Product<T> out = product<T>(h, F, w_out, F, N, C, F, y);
  if (few_tokens(N, C, F, dtype)) {
    launch_few<T, true>(in, dtype, nullptr, st);
    launch_few<T, false>(out, dtype, ws, st);
  } else {
    launch_product<T, kGated, false, false>(in, dtype, ws, st);
    launch_product<T, kPlain, false, false>(out, dtype, ws, st);
  }
}

// Workspaces hold the splits of one product after the other, the backward's [da, du] before them.
size_t ffn_fwd_ws(int64_t N, int C, int F, int dtype) {
  return few_tokens(N, C, F, dtype) ? few_part_bytes(N, C, F, dtype) : std::max(cut_of(N, F, C, dtype, kGated).part_bytes(), cut_of(N, C, F, dtype, kPlain).part_bytes());
}
size_t ffn_bwd_part(int64_t N, int F, int dtype) { return round_up((size_t)N * 2 * F * elem_size(dtype), 256); }
size_t ffn_bwd_ws(int64_t N, int C, int F, int dtype) {
  const int64_t F2 = 2 * (int64_t)F;
  return ffn_bwd_part(N, F, dtype) + std::max({cut_of(N, F, C, dtype, kGatedBwd).part_bytes(), cut_of(N, C, F2, dtype, kPlain).part_bytes(),
                                               cut_of(F2, C, N, dtype, kPlain).part_bytes(), cut_of(C, F, N, dtype, kPlain).part_bytes(),
                                               cut_of({{F2, C}, {C, F}}, N, dtype, kPlain).part_bytes()});
}

// What is enough for any number of tokens up to N: the splits of a call depend on how many tiles are behind its last whole round.
size_t ffn_fwd_room(int64_t N, int C, int F, int dtype) {
  return std::max({few_part_bytes(std::min<int64_t>(N, kFewTokens), C, F, dtype), most_part_bytes(N, F, C, dtype, kGated), most_part_bytes(N, C, F, dtype, kPlain)});
}
size_t ffn_bwd_room(int64_t N, int C, int F, int dtype) {
  const int64_t F2 = 2 * (int64_t)F;
  return ffn_bwd_part(N, F, dtype) + std::max({most_part_bytes(N, F, C, dtype, kGatedBwd), most_part_bytes(N, C, F2, dtype, kPlain), most_part_bytes_k({{F2, C}}, N, dtype),
                                               most_part_bytes_k({{C, F}}, N, dtype), most_part_bytes_k({{F2, C}, {C, F}}, N, dtype)});
}

template <typename T>
void ffn_bwd(const void* d_y, const void* x, const void* w_in, const void* w_out, const void* au, const void* h, int dtype, int64_t N, int C, int F,
             int act, void* d_x, void* d_w_in, void* d_w_out, void* ws, hipStream_t st) {
  void* part = (char*)ws + ffn_bwd_part(N, F, dtype);
  if (d_x || d_w_in) {
    Product<T> dh = product<T>(d_y, C, w_out, F, N, F, C, ws);
    dh.saved = (const T*)au;
    dh.act = act;
    launch_product<T, kGatedBwd, false, true>(dh, dtype, part, st);
  }
  if (d_x) launch_product<T, kPlain, false, true>(product<T>(ws, 2 * (int64_t)F, w_in, C, N, C, 2 * (int64_t)F, d_x), dtype, part, st);
  const Product<T> w_in_grad = product<T>(ws, 2 * (int64_t)F, x, C, 2 * (int64_t)F, C, N, d_w_in), w_out_grad = product<T>(d_y, C, h, F, C, F, N, d_w_out);
  if (d_w_in && d_w_out) launch_two<T, true, true>(w_in_grad, w_out_grad, dtype, part, st);
  else if (d_w_in) launch_product<T, kPlain, true, true>(w_in_grad, dtype, part, st);
  else if (d_w_out) launch_product<T, kPlain, true, true>(w_out_grad, dtype, part, st);
}

int check_ffn(int64_t N, int C, int F, int dtype, int act, bool backward) {
  if (N < 0 || C < 1 || F < 1) return MOGA_ERR_INVALID_ARG;
  if (dtype != MOGA_F32 && dtype != MOGA_BF16) return MOGA_ERR_UNSUPPORTED;
  if (act != MOGA_ACT_SILU && act != MOGA_ACT_GELU && act != MOGA_ACT_GELU_TANH) return MOGA_ERR_UNSUPPORTED;
  const int v = dtype == MOGA_F32 ? 4 : 8;
  if (C % v || F % v || C > kFfnMaxC || F > kFfnMaxF || N >= ((int64_t)1 << 31)) return MOGA_ERR_UNSUPPORTED;
  const int64_t F2 = 2 * (int64_t)F;
  // sizes whose smallest tiles fit, whichever are taken, else those that are
  const int64_t most = std::max({ceil_div(N, 64) * ceil_div(F, 64), ceil_div(N, 64) * ceil_div(C, 128), ceil_div(F2, 64) * ceil_div(C, 128), ceil_div(C, 64) * ceil_div(F, 128)});
  if (grid_fits(most + kMostSplits * 768, 512)) return MOGA_OK;
  const auto fits = [&](int64_t M, int64_t n, int64_t K, Kind kind) { return cut_of(M, n, K, dtype, kind).fits(); };
  if (backward) return fits(N, F, C, kGatedBwd) && fits(N, C, F2, kPlain) && fits(F2, C, N, kPlain) && fits(C, F, N, kPlain) ? MOGA_OK : MOGA_ERR_UNSUPPORTED;
  return fits(N, F, C, kGated) && fits(N, C, F, kPlain) ? MOGA_OK : MOGA_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace moga

using namespace moga;

extern "C" void moga_debug_set_ffn_tiles(int shape, int round, int splits, int together) {
  const bool on = shape >= 0 && shape < 3 && round > 0 && splits > 0 && splits <= kMostSplits;
  g_forced.store(on ? (long long)round << 24 | (together ? 1 : 0) << 16 | splits << 8 | (shape + 1) : 0);
}

extern "C" size_t moga_gated_ffn_fwd_ws_bytes(int64_t N, int C, int F, int dtype) {
  return check_ffn(N, C, F, dtype, MOGA_ACT_SILU, false) == MOGA_OK && N > 0 ? ffn_fwd_ws(N, C, F, dtype) : 0;
}
extern "C" size_t moga_gated_ffn_bwd_ws_bytes(int64_t N, int C, int F, int dtype) {
  return check_ffn(N, C, F, dtype, MOGA_ACT_SILU, true) == MOGA_OK && N > 0 ? ffn_bwd_ws(N, C, F, dtype) : 0;
}

extern "C" size_t moga_gated_ffn_fwd_preferred(int64_t N, int C, int F, int dtype) {
  return check_ffn(N, C, F, dtype, MOGA_ACT_SILU, false) == MOGA_OK && N > 0 ? ffn_fwd_room(N, C, F, dtype) : 0;
}
extern "C" size_t moga_gated_ffn_bwd_preferred(int64_t N, int C, int F, int dtype) {
  return check_ffn(N, C, F, dtype, MOGA_ACT_SILU, true) == MOGA_OK && N > 0 ? ffn_bwd_room(N, C, F, dtype) : 0;
}

extern "C" int moga_gated_ffn_fwd(const void* x, const void* w_in, const void* w_out, int dtype, int64_t N, int C, int F, int activation, void* h,
                                  void* au, void* y, void* ws, size_t ws_bytes, void* stream) {
  const int bad = check_ffn(N, C, F, dtype, activation, false);
  if (bad) return bad;
  if (N == 0) return MOGA_OK;
  if (!x || !w_in || !w_out || !h || !y) return MOGA_ERR_INVALID_ARG;
  if (!(aligned16(x) && aligned16(w_in) && aligned16(w_out) && aligned16(h) && aligned16(au) && aligned16(y) && aligned16(ws)))
    return MOGA_ERR_INVALID_ARG;
  const size_t need = moga_gated_ffn_fwd_ws_bytes(N, C, F, dtype);
  if (need && (!ws || ws_bytes < need)) return MOGA_ERR_WORKSPACE;
  const hipStream_t st = (hipStream_t)stream;
  if (dtype == MOGA_F32) ffn_fwd<float>(x, w_in, w_out, dtype, N, C, F, activation, h, au, y, ws, st);
  else ffn_fwd<unsigned short>(x, w_in, w_out, dtype, N, C, F, activation, h, au, y, ws, st);
  return launch_status();
}

extern "C" int moga_gated_ffn_bwd(const void* d_y, const void* x, const void* w_in, const void* w_out, const void* au, const void* h, int dtype,
                                  int64_t N, int C, int F, int activation, void* d_x, void* d_w_in, void* d_w_out, void* ws, size_t ws_bytes,
                                  void* stream) {
  const int bad = check_ffn(N, C, F, dtype, activation, true);
  if (bad) return bad;
  if (!(aligned16(d_y) && aligned16(x) && aligned16(w_in) && aligned16(w_out) && aligned16(au) && aligned16(h) && aligned16(d_x) &&
        aligned16(d_w_in) && aligned16(d_w_out) && aligned16(ws)))
    return MOGA_ERR_INVALID_ARG;
  const hipStream_t st = (hipStream_t)stream;
  if (N == 0) {   // of no tokens: zeros
    const int64_t floats = (int64_t)C * F * elem_size(dtype) / 4;   // C and F are multiples of 4
    if (d_w_in) launch_fill_zero((float*)d_w_in, 2 * floats, st);
    if (d_w_out) launch_fill_zero((float*)d_w_out, floats, st);
    return d_w_in || d_w_out ? launch_status() : MOGA_OK;
  }
  if (!d_x && !d_w_in && !d_w_out) return MOGA_OK;
  if (!d_y || ((d_x || d_w_in) && (!w_out || !au)) || (d_x && !w_in) || (d_w_in && !x) || (d_w_out && !h)) return MOGA_ERR_INVALID_ARG;
  if (!ws || ws_bytes < moga_gated_ffn_bwd_ws_bytes(N, C, F, dtype)) return MOGA_ERR_WORKSPACE;
  if (dtype == MOGA_F32) ffn_bwd<float>(d_y, x, w_in, w_out, au, h, dtype, N, C, F, activation, d_x, d_w_in, d_w_out, ws, st);
  else ffn_bwd<unsigned short>(d_y, x, w_in, w_out, au, h, dtype, N, C, F, activation, d_x, d_w_in, d_w_out, ws, st);
  return launch_status();
}
