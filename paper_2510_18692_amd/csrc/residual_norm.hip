// The residual sum of a block with its gate, and the norms before and after it, forward and backward.
//
//   z = post(y) post_weight,  r = x + residual_scale gate z,  h = (pre(r) weight + bias) (1 + scale) + shift
// post and pre are RMS or layer norms of a row (or nothing); gate, scale and shift have a row for every `tokens_per_row` tokens.  With
// G = residual_scale gate post_weight, W = weight (1 + scale), rh and yh the normalised rows, the backward of a token is
//   g = d_h W,  D = d_r + rstd (g - [mean g] - rh mean(g rh)) = d_x,  e = D G,  d_y = rstd_y (e - [mean e] - yh mean(e yh))
// ([]: of layer norms), and every parameter's gradient follows from three sums over the tokens of a row of the gate, column by column:
//   A1 = sum d_h, A2 = sum d_h rh, B = sum D yh:  d_shift = A1, d_scale = weight A2 + bias A1, d_gate = residual_scale post_weight B, and over all
//   rows d_weight = sum (1 + scale) A2, d_bias = sum (1 + scale) A1, d_post_weight = residual_scale sum gate B.
//
// Bound by HBM: the forward reads x and y and writes r and h, the backward reads x, y, d_r and d_h and writes d_x and d_y, each once; r is computed
// again from x and y, which are there, and so in 32 bits, while a stored r is rounded.  A row stays in registers between its two norms (two passes over
// them, mean and then centred squares), the next row is on its way, and the shares of the parameters' gradients stay there from token to token.
// 99,840 x 5120 bf16, RMS norms before and after: forward 832 us (4.9 TB/s of what it moves), backward 1,239 (4.9), its sums 9; 32,760 x 1536, stream fp32,
// block bf16, 21 rows of the gate: 116 (5.2), 196 (4.6) and 11; 4,099 x 1535 fp32, rows that start at any 4 bytes: 25, 33, 8 and 4.  torch's copy reaches 4.8.
// Beyond 8,192 columns a lane has two pieces of a row, and the backward's six rows of values do not fit its registers: 6,103 x 16384 bf16 1.54 ms, 0.78 TB/s.
#include <algorithm>
#include <cmath>

#include "norm_rows.h"

namespace moga {
namespace {

struct ResNorm {
  const void *x, *y;
  const float *gate, *post_weight, *weight, *bias, *scale, *shift;
  int64_t N, each;   // tokens; tokens of a row of gate, scale and shift
  int C, post, pre;
  float alpha, eps;
  // tokens are dealt out in pieces of `len` within a row of the gate
  int64_t pieces, items, len;
};

constexpr int kBlockWaves = 16;   // of a block that owns a token, at most

// Eight columns of a row.  EVEN: rows are whole eights, and a lane has all of one or none; else the row's last piece is looked at column by column
// (10^8 values bf16, backward: C 264 595 us so and 312 even, C 768 477 and 289, C 1000 380 and 284).
// The values stay as they lie until get(): without the asm the compiler unpacks them right behind the loads, for which the next row's do not have the
// registers (backward of 10^8 values bf16, C 5120: 597 us).
template <typename T, bool EVEN> struct Eight;
template <bool EVEN> struct Eight<unsigned short, EVEN> {
  Bytes16<unsigned short> b;
  __device__ __forceinline__ void load(const unsigned short* row, int col, int C, bool last) {
    if constexpr (EVEN) b = col < C ? *(const Bytes16<unsigned short>*)(row + col) : Bytes16<unsigned short>{};
    else b = load_part(row, col, C, last);
  }
  __device__ __forceinline__ void get(float (&f)[8], int col, int C) {
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("" : "+v"(b.w[i]));
    unpack(b, f);
    if constexpr (!EVEN) clear_past(f, col, C);
  }
};
template <bool EVEN> struct Eight<float, EVEN> {
  Bytes16<float> b[2];
  __device__ __forceinline__ void load(const float* row, int col, int C, bool last) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (EVEN) b[i] = col < C ? *(const Bytes16<float>*)(row + col + 4 * i) : Bytes16<float>{};
      else b[i] = load_part(row, col + 4 * i, C, last);
    }
  }
  __device__ __forceinline__ void get(float (&f)[8], int col, int C) {
#pragma unroll
    for (int i = 0; i < 8; ++i) asm("" : "+v"(b[i / 4].w[i % 4]));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(b[i / 4].w[i % 4]);
    if constexpr (!EVEN) clear_past(f, col, C);
  }
};
template <bool EVEN>
__device__ __forceinline__ void store8(unsigned short* row, int col, int C, const float (&f)[8]) {
  if constexpr (!EVEN) store_part(row, col, C, f);
  else if (col < C) *(Bytes16<unsigned short>*)(row + col) = pack(f);
}
template <bool EVEN>
__device__ __forceinline__ void store8(float* row, int col, int C, const float (&f)[8]) {
  const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
  if constexpr (!EVEN) {
    store_part(row, col, C, lo);
    store_part(row, col + 4, C, hi);
  } else if (col < C) {
    *(Bytes16<float>*)(row + col) = pack(lo);
    *(Bytes16<float>*)(row + col + 4) = pack(hi);
  }
}

// Eight floats of a lane's own between tokens, in LDS: the registers go to more waves.  99,840 x 5120 bf16, RMS norms before and after: 869 us with the
// forward's three factors there, 947 in registers; the backward gains nothing.
struct Parked {
  floatx4_t* at;   // [2][threads], of this lane
  int threads;
  __device__ __forceinline__ Parked(floatx4_t* lds, int slot) : at(lds + (size_t)slot * 2 * blockDim.x + threadIdx.x), threads(blockDim.x) {}
  __device__ __forceinline__ void put(const float (&v)[8]) const {
    at[0] = floatx4_t{v[0], v[1], v[2], v[3]};
    at[threads] = floatx4_t{v[4], v[5], v[6], v[7]};
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const floatx4_t a = at[0], b = at[threads];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
};

// How the tokens of a piece are dealt out: LANES = 8 to 64 to a token, four waves a block; LANES = 0: a token to a block.
template <int LANES>
struct Lanes {
  static constexpr int kRows = LANES ? 256 / LANES : 1;
  int lanes, lane, slot;
  __device__ __forceinline__ Lanes() {
    lanes = LANES ? LANES : blockDim.x;
    lane = LANES ? threadIdx.x % LANES : threadIdx.x;
    slot = LANES ? threadIdx.x / LANES : 0;
  }
};

// Tokens [first, end) of a piece, all of the same row of the gate.
struct Piece {
  int64_t row, first, end;
  __device__ __forceinline__ Piece(const ResNorm& p, int64_t item) {
    row = item / p.pieces;
    const int64_t a = row * p.each;
    first = a + (item - row * p.pieces) * p.len;
    end = min(min(a + p.each, p.N), first + p.len);
  }
};

// G and W of eight columns, for one row of gate, scale and shift.
__device__ __forceinline__ void load_factors(const ResNorm& p, int64_t row, int col, float (&G)[8], float (&W)[8]) {
  float t[8];
  load_weights(p.gate ? p.gate + row * p.C : nullptr, col, p.C, 1.f, G);
  load_weights(p.post_weight, col, p.C, 1.f, t);
#pragma unroll
  for (int i = 0; i < 8; ++i) G[i] *= p.alpha * t[i];
  load_weights(p.weight, col, p.C, 1.f, W);
  load_weights(p.scale ? p.scale + row * p.C : nullptr, col, p.C, 0.f, t);
#pragma unroll
  for (int i = 0; i < 8; ++i) W[i] *= 1.f + t[i];
}

// Mean (0 of an RMS norm) and 1 / deviation of a row; v is centred.  Columns past the row's end are 0 and stay 0.
template <int PARTS, typename Sum>
__device__ __forceinline__ void row_stats(float (&v)[PARTS][8], int kind, int C, const int (&col)[PARTS], float n, float eps, Sum& sum, float& mu,
                                          float& rstd) {
  float s[1];
  mu = 0.f;
  if (kind == MOGA_NORM_LAYER) {
    s[0] = 0.f;
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[q][i];
    sum(s);
    mu = s[0] / n;
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[q][i] = col[q] + i < C ? v[q][i] - mu : 0.f;
  }
  s[0] = 0.f;
#pragma unroll
  for (int q = 0; q < PARTS; ++q)
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] = fmaf(v[q][i], v[q][i], s[0]);
  sum(s);
  rstd = 1.f / sqrtf(s[0] / n + eps);
}

// TX: x and r; TY: y and h.  PARTS pieces of eight columns a lane; lane t holds the columns (part * lanes + t) * 8 ..
template <typename TX, typename TY, int LANES, int PARTS, int WAVES, bool EVEN>
__global__ __launch_bounds__(64 * WAVES, WAVES > 4 && PARTS == 1 ? 5 : 4) void residual_norm_fwd_kernel(const ResNorm p, TX* __restrict__ r_out, TY* __restrict__ h_out,
                                                                                        float* __restrict__ stats) {
  __shared__ float lds[2][WAVES][1];
  RowSum<LANES, 1, WAVES> sum{lds};
  const Lanes<LANES> d;
  const TX* x = (const TX*)p.x;
  const TY* y = (const TY*)p.y;
  const int C = p.C;
  const float n = (float)C;
  int col[PARTS];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) col[q] = (q * d.lanes + d.lane) * 8;
  // G, W and the additive term; of two pieces a lane they would take more LDS than there is
  constexpr bool PARKED = PARTS == 1;
  extern __shared__ floatx4_t s_kept[];
  float kept[PARKED ? 1 : PARTS][3][8];
  auto keep = [&](int q, int k, const float (&v)[8]) {
    if constexpr (PARKED) {
      Parked(s_kept, k).put(v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) kept[q][k][i] = v[i];
    }
  };
  auto recall = [&](int q, int k, float (&v)[8]) {
    if constexpr (PARKED) {
      Parked(s_kept, k).get(v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = kept[q][k][i];
    }
  };
  int64_t held = -1;
  for (int64_t item = blockIdx.x; item < p.items; item += gridDim.x) {
    const Piece piece(p, item);
    int64_t row = piece.first + d.slot;
    Eight<TX, EVEN> nx[PARTS];
    Eight<TY, EVEN> ny[PARTS];
    auto fetch = [&](int64_t at) {
#pragma unroll
      for (int q = 0; q < PARTS; ++q) nx[q].load(x + at * C, col[q], C, at + 1 == p.N);
      if (y)
#pragma unroll
        for (int q = 0; q < PARTS; ++q) ny[q].load(y + at * C, col[q], C, at + 1 == p.N);
    };
    if (row < piece.end) fetch(row);
    if (held != piece.row) {
      held = piece.row;
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        float G[8], W[8], S[8], t[8];
        load_factors(p, held, col[q], G, W);
        keep(q, 0, G);
        keep(q, 1, W);
        load_weights(p.scale ? p.scale + held * C : nullptr, col[q], C, 0.f, t);
        load_weights(p.bias, col[q], C, 0.f, S);
#pragma unroll
        for (int i = 0; i < 8; ++i) S[i] *= 1.f + t[i];
        load_weights(p.shift ? p.shift + held * C : nullptr, col[q], C, 0.f, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) S[i] += t[i];
        keep(q, 2, S);
      }
    }
    for (; row < piece.end; row += Lanes<LANES>::kRows) {
      float f[PARTS][8], v[PARTS][8];
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        nx[q].get(f[q], col[q], C);
        if (y) {
          ny[q].get(v[q], col[q], C);
        }
      }
      if (row + Lanes<LANES>::kRows < piece.end) fetch(row + Lanes<LANES>::kRows);
      float mu = 0.f, rstd = 1.f;
      if (y) {
        if (p.post != MOGA_NORM_NONE) {
          row_stats(v, p.post, C, col, n, p.eps, sum, mu, rstd);
          if (stats && d.lane == 0) {
            stats[row] = mu;
            stats[p.N + row] = rstd;
          }
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
          float G[8];
          recall(q, 0, G);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[q][i] = fmaf(v[q][i] * rstd, G[i], f[q][i]);
          store8<EVEN>(r_out + row * C, col[q], C, f[q]);
        }
      }
      if (p.pre != MOGA_NORM_NONE) {
        row_stats(f, p.pre, C, col, n, p.eps, sum, mu, rstd);
        if (stats && d.lane == 0) {
          stats[2 * p.N + row] = mu;
          stats[3 * p.N + row] = rstd;
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
          float W[8], S[8];
          recall(q, 1, W);
          recall(q, 2, S);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[q][i] = fmaf(f[q][i] * rstd, W[i], S[i]);
          store8<EVEN>(h_out + row * C, col[q], C, f[q]);
        }
      }
    }
  }
}

struct ResNormGrads {
  const void *d_r, *d_h;
  const float* stats;
  void *d_x, *d_y;
  float* part;   // [items][3][C]: A1, A2, B, or NULL
};

// The shares of the tokens that run beside each other in a block are added in a fixed order: results repeat bit by bit.
// Three waves a SIMD; of blocks of three waves, of which a CU takes four only where each SIMD has room for one wave more, four (10^8 values, C 1536: bf16 282 us
// instead of 325, stream fp32 401 instead of 433; the other blocks lose up to a tenth so, fp32 alone gains nothing).
template <typename TX, typename TY, int LANES, int PARTS, int WAVES, bool EVEN>
__global__ __launch_bounds__(64 * WAVES, WAVES > 4 || (WAVES == 3 && sizeof(TY) == 2) ? 4 : 3) void residual_norm_bwd_kernel(const ResNorm p, const ResNormGrads o) {
#pragma clang fp contract(off)   // g is one value in its mean and in what the mean is taken from
  __shared__ float lds[2][WAVES][2];
  RowSum<LANES, 2, WAVES> sum{lds};
  const Lanes<LANES> d;
  const TX *x = (const TX*)p.x, *dr = (const TX*)o.d_r;
  const TY *y = (const TY*)p.y, *dh = (const TY*)o.d_h;
  const int C = p.C;
  const float n = (float)C;
  const bool post = p.post != MOGA_NORM_NONE;
  int col[PARTS];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) col[q] = (q * d.lanes + d.lane) * 8;
  float G[PARTS][8], W[PARTS][8];
  int64_t held = -1;
  for (int64_t item = blockIdx.x; item < p.items; item += gridDim.x) {
    const Piece piece(p, item);
    int64_t row = piece.first + d.slot;
    Eight<TX, EVEN> nx[PARTS], nr[PARTS];
    Eight<TY, EVEN> ny[PARTS], nh[PARTS];
    float st[4];
    auto fetch = [&](int64_t at) {
      const bool last = at + 1 == p.N;
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        if (dh) {
          nx[q].load(x + at * C, col[q], C, last);
          nh[q].load(dh + at * C, col[q], C, last);
        }
        if (y) ny[q].load(y + at * C, col[q], C, last);
        if (dr) nr[q].load(dr + at * C, col[q], C, last);
      }
      if (y && post) {
        st[0] = o.stats[at];
        st[1] = o.stats[p.N + at];
      }
      if (dh) {
        st[2] = o.stats[2 * p.N + at];
        st[3] = o.stats[3 * p.N + at];
      }
    };
    if (row < piece.end) fetch(row);
    if (held != piece.row) {
      held = piece.row;
#pragma unroll
      for (int q = 0; q < PARTS; ++q) load_factors(p, held, col[q], G[q], W[q]);
    }
    float a1[PARTS][8], a2[PARTS][8], bs[PARTS][8];
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) a1[q][i] = a2[q][i] = bs[q][i] = 0.f;
    for (; row < piece.end; row += Lanes<LANES>::kRows) {
      float f[PARTS][8], v[PARTS][8], D[PARTS][8], g[PARTS][8];
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        if (dh) {
          nx[q].get(f[q], col[q], C);
          nh[q].get(g[q], col[q], C);
        }
        if (y) {
          ny[q].get(v[q], col[q], C);
        }
        if (dr) {
          nr[q].get(D[q], col[q], C);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) D[q][i] = 0.f;
        }
      }
      const float mu_y = post ? st[0] : 0.f, r_y = post ? st[1] : 1.f, mu = st[2], r = st[3];
      if (row + Lanes<LANES>::kRows < piece.end) fetch(row + Lanes<LANES>::kRows);
      if (y) {
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[q][i] = (v[q][i] - mu_y) * r_y;   // past the row's end its products are with zeros
      }
      if (dh) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (y) f[q][i] = fmaf(v[q][i], G[q][i], f[q][i]);
            f[q][i] = (f[q][i] - mu) * r;
            a1[q][i] += g[q][i];
            a2[q][i] = fmaf(g[q][i], f[q][i], a2[q][i]);
            g[q][i] *= W[q][i];
            s[0] += g[q][i];
            s[1] = fmaf(g[q][i], f[q][i], s[1]);
          }
        sum(s);
        const float m0 = p.pre == MOGA_NORM_LAYER ? s[0] / n : 0.f, m1 = s[1] / n;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            D[q][i] += r * (g[q][i] - m0 - f[q][i] * m1);
            if (EVEN) D[q][i] = col[q] < C ? D[q][i] : 0.f;
          }
          if constexpr (!EVEN) clear_past(D[q], col[q], C);
        }
      }
#pragma unroll
      for (int q = 0; q < PARTS; ++q) store8<EVEN>((TX*)o.d_x + row * C, col[q], C, D[q]);
      if (y) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            bs[q][i] = fmaf(D[q][i], v[q][i], bs[q][i]);
            D[q][i] *= G[q][i];
            s[0] += D[q][i];
            s[1] = fmaf(D[q][i], v[q][i], s[1]);
          }
        if (post) {
          sum(s);
          const float m0 = p.post == MOGA_NORM_LAYER ? s[0] / n : 0.f, m1 = s[1] / n;
#pragma unroll
          for (int q = 0; q < PARTS; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) D[q][i] = r_y * (D[q][i] - m0 - v[q][i] * m1);
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) store8<EVEN>((TY*)o.d_y + row * C, col[q], C, D[q]);
      }
    }
    if (!o.part) continue;
    float* out = o.part + item * 3 * C;
    if constexpr (LANES == 0) {
#pragma unroll
      for (int q = 0; q < PARTS; ++q)
        if (col[q] + 8 <= C) {
          store8<true>(out, col[q], C, a1[q]);
          store8<true>(out + C, col[q], C, a2[q]);
          store8<true>(out + 2 * C, col[q], C, bs[q]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (col[q] + i < C) {
              out[col[q] + i] = a1[q][i];
              out[C + col[q] + i] = a2[q][i];
              out[2 * C + col[q] + i] = bs[q][i];
            }
        }
    } else {
      __shared__ float acc[3][LANES * PARTS * 8];
      const int wave = threadIdx.x >> 6;
      if constexpr (LANES < 64) {   // the tokens of a wave
        auto all = [](float t) {
          int v = __float_as_int(t);
          if constexpr (LANES <= 8) v = combine_xor<8>(v, AddF{});
          if constexpr (LANES <= 16) v = combine_xor<16>(v, AddF{});
          return __int_as_float(combine_xor<32>(v, AddF{}));
        };
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            a1[q][i] = all(a1[q][i]);
            a2[q][i] = all(a2[q][i]);
            bs[q][i] = all(bs[q][i]);
          }
      }
      __syncthreads();   // the last item's sums are read
      for (int k = 0; k < 4; ++k) {
        if (wave == k && (threadIdx.x & 63) < LANES) {
#pragma unroll
          for (int q = 0; q < PARTS; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              acc[0][col[q] + i] = k == 0 ? a1[q][i] : acc[0][col[q] + i] + a1[q][i];
              acc[1][col[q] + i] = k == 0 ? a2[q][i] : acc[1][col[q] + i] + a2[q][i];
              acc[2][col[q] + i] = k == 0 ? bs[q][i] : acc[2][col[q] + i] + bs[q][i];
            }
        }
        __syncthreads();
      }
      for (int c = threadIdx.x; c < C; c += 256)
#pragma unroll
        for (int k = 0; k < 3; ++k) out[k * C + c] = acc[k][c];
    }
  }
}

struct ResNormSums {
  float *d_gate, *d_post_weight, *d_weight, *d_bias, *d_scale, *d_shift;   // each may be NULL
  float* over;   // [groups][3][C]: weighted sums of the rows of a group of blocks, where there are several groups
};

// Sums over the pieces of each row of the gate, in a fixed order: 16 columns a block, whose 16 threads each take every 16th piece; rows in `gridDim.y`
// groups.  Bound by its chain of loads: of 32 columns and 8 threads, with whole lines, it takes a third longer.
__global__ __launch_bounds__(256) void residual_norm_sums_kernel(const ResNorm p, const float* __restrict__ part, const ResNormSums o, int64_t rows) {
  __shared__ float acc[3][16][17];
  const int c = threadIdx.x & 15, k = threadIdx.x >> 4, C = p.C;
  const int col = blockIdx.x * 16 + c;
  const float w = p.weight && col < C ? p.weight[col] : 1.f, b = p.bias && col < C ? p.bias[col] : 0.f;
  const float wp = p.post_weight && col < C ? p.post_weight[col] : 1.f;
  float all[3] = {0.f, 0.f, 0.f};
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    constexpr int U = 4;   // loads of each on their way
    float s[3][U];
#pragma unroll
    for (int u = 0; u < U; ++u) s[0][u] = s[1][u] = s[2][u] = 0.f;
    // pieces past the last token were not written
    const int64_t tokens = min(p.each, p.N - row * p.each), used = (tokens + p.len - 1) / p.len;
    if (col < C)
      for (int64_t i = k; i < used; i += 16 * U)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + 16 * u < used) {
            const float* at = part + (row * p.pieces + i + 16 * u) * 3 * C + col;
            s[0][u] += at[0];
            s[1][u] += at[C];
            s[2][u] += at[2 * C];
          }
#pragma unroll
    for (int h = U / 2; h > 0; h /= 2)
#pragma unroll
      for (int u = 0; u < h; ++u)
#pragma unroll
        for (int j = 0; j < 3; ++j) s[j][u] += s[j][u + h];
#pragma unroll
    for (int j = 0; j < 3; ++j) acc[j][k][c] = s[j][0];
    __syncthreads();
    if (k == 0 && col < C) {
      float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int j = 0; j < 3; ++j) t[j] += acc[j][i][c];
      const int64_t at = row * C + col;
      if (o.d_shift) o.d_shift[at] = t[0];
      if (o.d_scale) o.d_scale[at] = fmaf(w, t[1], b * t[0]);
      if (o.d_gate) o.d_gate[at] = p.alpha * wp * t[2];
      const float up = p.scale ? 1.f + p.scale[at] : 1.f, gate = p.gate ? p.gate[at] : 1.f;
      all[0] = fmaf(up, t[0], all[0]);
      all[1] = fmaf(up, t[1], all[1]);
      all[2] = fmaf(p.alpha * gate, t[2], all[2]);
    }
    __syncthreads();
  }
  if (k == 0 && col < C) {
    if (gridDim.y > 1) {
#pragma unroll
      for (int j = 0; j < 3; ++j) o.over[((int64_t)blockIdx.y * 3 + j) * C + col] = all[j];
    } else {
      if (o.d_bias) o.d_bias[col] = all[0];
      if (o.d_weight) o.d_weight[col] = all[1];
      if (o.d_post_weight) o.d_post_weight[col] = all[2];
    }
  }
}

// Sums over the groups of rows.
__global__ __launch_bounds__(256) void residual_norm_over_kernel(const float* __restrict__ over, int groups, int C, const ResNormSums o) {
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= C) return;
  float s[3] = {0.f, 0.f, 0.f};
#pragma unroll 4
  for (int g = 0; g < groups; ++g)
#pragma unroll
    for (int j = 0; j < 3; ++j) s[j] += over[((int64_t)g * 3 + j) * C + col];
  if (o.d_bias) o.d_bias[col] = s[0];
  if (o.d_weight) o.d_weight[col] = s[1];
  if (o.d_post_weight) o.d_post_weight[col] = s[2];
}

// 8 columns a lane up to 8,192: a token goes to 8 lanes up to 64 columns, 16 up to 128, 32 up to 256, a wave up to 512, else to a block of a wave per 512.
// Lanes without columns are bytes that are not on their way: 10^8 values bf16, C 64 by 8 lanes 176 us forward and 298 backward, by 16 186 and 672 (before the
// even form); what is left of it, C 264 178 and 312, C 520 184 and 382.
struct Shape {
  int lanes, parts, waves, rows;
};
Shape shape_of(int C) {
  for (int lanes = 8; lanes <= 64; lanes *= 2)
    if (C <= 8 * lanes) return {lanes, 1, 4, 256 / lanes};
  return {0, C <= 8192 ? 1 : 2, std::min(kBlockWaves, (C + 511) / 512), 1};
}

constexpr int kOverGroups = 64;   // groups of gate rows whose weighted sums are added up by a kernel of their own

bool has_rows(const moga_residual_norm* a) { return a->gate || a->scale || a->shift; }

// Pieces: as many as fill the chip, of no fewer than `least` tokens a lane group.
void deal(ResNorm& p, int64_t rows, int blocks, int least, bool sums) {
  const Shape s = shape_of(p.C);
  const int64_t tokens = std::min(p.each, p.N), most = std::max<int64_t>(1, tokens / ((int64_t)s.rows * least));
  // one round of blocks for one row, and of the backward, whose pieces leave sums, where each row gets four or more; else rounds enough that the last
  // one is short
  p.pieces = std::min(most, rows == 1 || (sums && blocks / rows >= 4) ? blocks / rows : (4 * blocks + rows - 1) / rows);
  p.len = (tokens + p.pieces - 1) / p.pieces;
  p.pieces = (tokens + p.len - 1) / p.len;
  p.items = (rows - 1) * p.pieces + (p.N - (rows - 1) * p.each + p.len - 1) / p.len;   // none past the last token
}
int blocks_of(const Shape& s, int waves) { return 256 * std::max(1, waves / s.waves); }

ResNorm make(const moga_residual_norm* a) {
  const int64_t each = has_rows(a) && a->N > 0 ? std::min(a->tokens_per_row, a->N) : std::max<int64_t>(a->N, 1);
  return {a->x, a->y, a->gate, a->post_weight, a->weight, a->bias, a->scale, a->shift, a->N, each, a->C, a->y ? a->post : MOGA_NORM_NONE, a->pre,
          a->residual_scale, a->eps, 1, 1, 1};
}
constexpr int kFwdWaves = 24, kBwdWaves = 12;   // of a CU
// Tokens of a lane group and piece, of the backward: a piece's tokens take their turns, and so do the pieces whose sums are added up, 64 at a time.  With
// k tokens of each of a block's s.rows lane groups that is k turns and N / (64 k s.rows) turns, fewest in all where the two are alike: k^2 = N / (64 s.rows).
// Few tokens go in shorter pieces: bf16, us with one row of the gate, pieces of 8 tokens and these: C 5120, 8 tokens 26 and 10, 300 31 and 22, 1,560 37 and 35;
// C 512, 63 tokens 24 and 9, 3,000 19 and 17, 8,000 23 and 25.
int bwd_least(int64_t N, const Shape& s) {
  int least = 1;
  while (least < 8 && (int64_t)least * least * 64 * s.rows < N) ++least;
  return least;
}

ResNorm make_bwd(const moga_residual_norm* a) {
  ResNorm p = make(a);
  if (a->N > 0) deal(p, (a->N + p.each - 1) / p.each, blocks_of(shape_of(p.C), kBwdWaves), bwd_least(a->N, shape_of(p.C)), true);
  return p;
}

bool a16(const void* p) { return aligned16(p); }

int check_residual_norm(const moga_residual_norm* a) {
  if (!a || a->N < 0 || a->C < 1) return MOGA_ERR_INVALID_ARG;
  if (a->x_dtype != MOGA_F32 && a->x_dtype != MOGA_BF16) return MOGA_ERR_UNSUPPORTED;
  if (a->y_dtype != a->x_dtype && !(a->x_dtype == MOGA_F32 && a->y_dtype == MOGA_BF16)) return MOGA_ERR_UNSUPPORTED;
  for (int k : {a->post, a->pre})
    if (k != MOGA_NORM_NONE && k != MOGA_NORM_RMS && k != MOGA_NORM_LAYER) return MOGA_ERR_UNSUPPORTED;
  if (a->C > kNormMaxC || a->N >= ((int64_t)1 << 31)) return MOGA_ERR_UNSUPPORTED;
  if (!(a->eps >= 0.f) || !(a->eps < INFINITY) || !std::isfinite(a->residual_scale)) return MOGA_ERR_INVALID_ARG;
  if (a->tokens_per_row < 1) return MOGA_ERR_INVALID_ARG;
  if (a->N == 0) return MOGA_OK;   // no tensor of tokens need be there
  if (!a->y && (a->gate || a->post_weight || a->post != MOGA_NORM_NONE)) return MOGA_ERR_INVALID_ARG;
  if (a->post == MOGA_NORM_NONE && a->post_weight) return MOGA_ERR_INVALID_ARG;
  if (a->pre == MOGA_NORM_NONE && (a->weight || a->bias || a->scale || a->shift || !a->y)) return MOGA_ERR_INVALID_ARG;
  if (!(a16(a->x) && a16(a->y) && a16(a->gate) && a16(a->post_weight) && a16(a->weight) && a16(a->bias) && a16(a->scale) && a16(a->shift)))
    return MOGA_ERR_INVALID_ARG;
  return MOGA_OK;
}

// f(lanes, parts, most waves of a block), as constants
template <typename F>
void with_shape(const Shape& s, F&& f) {
#define MOGA_SHAPE(L, P, W) f(std::integral_constant<int, L>{}, std::integral_constant<int, P>{}, std::integral_constant<int, W>{})
  if (s.lanes == 8) MOGA_SHAPE(8, 1, 4);
  else if (s.lanes == 16) MOGA_SHAPE(16, 1, 4);
  else if (s.lanes == 32) MOGA_SHAPE(32, 1, 4);
  else if (s.lanes == 64) MOGA_SHAPE(64, 1, 4);
  else if (s.waves == 3) MOGA_SHAPE(0, 1, 3);
  else if (s.waves <= 4) MOGA_SHAPE(0, 1, 4);
  else if (s.parts == 1) MOGA_SHAPE(0, 1, kBlockWaves);
  else MOGA_SHAPE(0, 2, kBlockWaves);
#undef MOGA_SHAPE
}
// f(x, y) with a value of either type
template <typename F>
void with_types(int x_dtype, int y_dtype, F&& f) {
  if (x_dtype == MOGA_BF16) f((unsigned short)0, (unsigned short)0);
  else if (y_dtype == MOGA_BF16) f(0.f, (unsigned short)0);
  else f(0.f, 0.f);
}

}  // namespace
}  // namespace moga

using namespace moga;

extern "C" int moga_residual_norm_fwd(const moga_residual_norm* a, void* r, void* h, float* stats, void* stream) {
  const int bad = check_residual_norm(a);
  if (bad) return bad;
  if (a->N == 0) return MOGA_OK;
  if (!a->x || (a->y && !r) || (a->pre != MOGA_NORM_NONE && !h)) return MOGA_ERR_INVALID_ARG;
  if (!(a16(r) && a16(h) && a16(stats))) return MOGA_ERR_INVALID_ARG;
  const Shape s = shape_of(a->C);
  ResNorm p = make(a);
  const int blocks = blocks_of(s, kFwdWaves);
  deal(p, (p.N + p.each - 1) / p.each, blocks, p.N > blocks * s.rows ? 3 : 1, false);   // 4,099 x 1535 fp32, three rows of the gate: pieces of one token 38 us, of three 27
  const unsigned grid = (unsigned)std::min<int64_t>(p.items, 8 * blocks);
  with_types(a->x_dtype, a->y_dtype, [&](auto tx, auto ty) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    with_shape(s, [&](auto lanes, auto parts, auto waves) {
      const unsigned lds = parts.value == 1 ? 64 * s.waves * 96 : 0;
      if (p.C % 8 == 0)
        residual_norm_fwd_kernel<TX, TY, lanes.value, parts.value, waves.value, true><<<grid, 64 * s.waves, lds, (hipStream_t)stream>>>(p, (TX*)r, (TY*)h, stats);
      else
        residual_norm_fwd_kernel<TX, TY, lanes.value, parts.value, waves.value, false><<<grid, 64 * s.waves, lds, (hipStream_t)stream>>>(p, (TX*)r, (TY*)h, stats);
    });
  });
  return launch_status();
}

// M: rows of gate, scale and shift.  deal() makes no more pieces than this: all but the last of each row are of bwd_least tokens a lane group or more.
// Fewer tokens need no more bytes, though bwd_least falls with them: pieces of k - 1 tokens are 64 (k - 1) at most.
extern "C" size_t moga_residual_norm_bwd_ws_bytes(int64_t N, int M, int C) {
  if (N <= 0 || M < 1 || M > N || C < 1 || C > kNormMaxC || N >= ((int64_t)1 << 31)) return 0;
  const Shape s = shape_of(C);
  const int least = bwd_least(N, s);
  const int64_t items = M + std::min<int64_t>(4 * blocks_of(s, kBwdWaves), std::max<int64_t>(N / (s.rows * least), 64 * (least - 1)));
  return ((size_t)items + kOverGroups) * 3 * C * sizeof(float);
}

extern "C" int moga_residual_norm_bwd(const moga_residual_norm* a, const float* stats, const void* d_r, const void* d_h, void* d_x, void* d_y,
                                      float* d_gate, float* d_post_weight, float* d_weight, float* d_bias, float* d_scale, float* d_shift, void* ws,
                                      size_t ws_bytes, void* stream) {
  const int bad = check_residual_norm(a);
  if (bad) return bad;
  const bool sums = d_gate || d_post_weight || d_weight || d_bias || d_scale || d_shift;
  if ((d_gate && !a->gate) || (d_post_weight && !a->post_weight) || (d_weight && !a->weight) || (d_bias && !a->bias) || (d_scale && !a->scale) ||
      (d_shift && !a->shift))
    return MOGA_ERR_INVALID_ARG;
  if (!(a16(stats) && a16(d_r) && a16(d_h) && a16(d_x) && a16(d_y) && a16(d_gate) && a16(d_post_weight) && a16(d_weight) && a16(d_bias) &&
        a16(d_scale) && a16(d_shift) && a16(ws)))
    return MOGA_ERR_INVALID_ARG;
  if (a->N == 0 && !sums) return MOGA_OK;
  const hipStream_t st = (hipStream_t)stream;
  ResNorm p = make_bwd(a);
  const int64_t rows = a->N ? (p.N + p.each - 1) / p.each : 1;
  if (a->N > 0) {
    const bool norms = a->pre != MOGA_NORM_NONE || a->post != MOGA_NORM_NONE;
    if (!a->x || !d_x || (a->y && !d_y) || (norms && !stats) || (a->pre != MOGA_NORM_NONE) != (d_h != nullptr)) return MOGA_ERR_INVALID_ARG;
    if (sums && (!ws || ws_bytes < moga_residual_norm_bwd_ws_bytes(p.N, (int)rows, p.C))) return MOGA_ERR_WORKSPACE;
    const Shape s = shape_of(p.C);
    const ResNormGrads o{d_r, d_h, stats, d_x, d_y, sums ? (float*)ws : nullptr};
    const unsigned grid = (unsigned)std::min<int64_t>(p.items, 8 * blocks_of(s, kBwdWaves));
    with_types(a->x_dtype, a->y_dtype, [&](auto tx, auto ty) {
      with_shape(s, [&](auto lanes, auto parts, auto waves) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        if (p.C % 8 == 0) residual_norm_bwd_kernel<TX, TY, lanes.value, parts.value, waves.value, true><<<grid, 64 * s.waves, 0, st>>>(p, o);
        else residual_norm_bwd_kernel<TX, TY, lanes.value, parts.value, waves.value, false><<<grid, 64 * s.waves, 0, st>>>(p, o);
      });
    });
  } else {
    p.N = 0;   // of no tokens: zeros
  }
  if (sums) {
    const int groups = (int)std::min<int64_t>(rows, kOverGroups);
    const ResNormSums o{d_gate, d_post_weight, d_weight, d_bias, d_scale, d_shift, (float*)ws + (size_t)p.items * 3 * p.C};
    residual_norm_sums_kernel<<<dim3((p.C + 15) / 16, groups), 256, 0, st>>>(p, (const float*)ws, o, rows);
    if (groups > 1 && (d_post_weight || d_weight || d_bias)) residual_norm_over_kernel<<<(p.C + 255) / 256, 256, 0, st>>>(o.over, groups, p.C, o);
  }
  return launch_status();
}
