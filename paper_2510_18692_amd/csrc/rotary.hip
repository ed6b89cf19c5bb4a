// Rotary positions of queries and keys, in token order or on the way into (and out of) the groups' order.
//
// The first R channels of a head are R / 2 pairs, neighbours (2 i, 2 i + 1) or (i, i + R / 2).  Pair i of a token at position p is
// turned by the angle p * inv_freq[i] and scaled:
//   y1 = f (x1 cos - x2 sin), y2 = f (x2 cos + x1 sin); the backward turns by minus the angle.
// With several axes a token has a position on each, and every axis a run of pairs.
// In maps (differential attention) each half of a head is turned by itself, as a head of D / 2 channels would be.
//
// Angles: the product and its reduction to a part of a turn in 64 bits (at position 500,000 a product in 32 bits is 0.03 radians off), then
// sine and cosine in 32 bits, once per token and pair, in LDS, for all heads of q and k.
//
// Bound by HBM: every chunk of 16 bytes is read and written once, by a lane of its own, so that loads and stores are whole rows.  A lane of the
// half layout reads its partner's chunk too, from L1; one lane for both partners halves those loads but splits every row's traffic in two:
// 32,760 x 12 heads of 128, 96 channels turned, bf16, into sorted order 139 us against 128, back 149 against 139.  Three chunks of a lane in
// flight together were slower everywhere (149, 156; fewer waves fit).  By itself each launch takes 132 and 140 us (4.6 and 4.3 TB/s), in maps of 64
// channels 132 and 141, in fp32 265 and 273; the call that moves the same rows back without turning them 122, this one 144.  In token order,
// neighbours, three axes, 99,840 x 40 heads of q and k, bf16 0.73 ms (5.6 TB/s), 49,920 x 40, fp32 0.76 (5.4).
#include <algorithm>
#include <cmath>

#include "moga_common.h"

namespace moga {
namespace {

constexpr int kMaxAxes = 4, kMaxHeadDim = 256;

template <typename T> struct Chunk;
template <> struct Chunk<float> {
  static constexpr int V = 4;
  __device__ static void get(uintx4_t w, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
  }
  __device__ static uintx4_t put(const float (&f)[4]) {
    return uintx4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <> struct Chunk<unsigned short> {
  static constexpr int V = 8;
  __device__ static void get(uintx4_t w, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_lo_to_f32(w[i]);
      f[2 * i + 1] = bf16_hi_to_f32(w[i]);
    }
  }
  __device__ static uintx4_t put(const float (&f)[8]) {   // to nearest even
    return uintx4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  }
};
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(unsigned short v) { return bf16_bits_to_f32(v); }

struct RotaryArgs {
  const void* src[3];   // q, k, v
  void* dst[3];
  int heads[3], first[4];   // heads of each; first[i]: those before it, first[3] of all
  const int32_t* pos;       // [axes][N]
  const double* inv_freq;   // [pairs]
  const int32_t* perm;      // sorted order: slot -> token
  int64_t N;
  int D, R, axes, bound[kMaxAxes];   // R: turned channels of a head, or of each map; bound[a]: pairs of the axes up to a
  int pairs, second;                 // pairs that have an angle; in maps: which of them is the second map's first
  float factor, sign;
  int tokens, heads_each;   // of a block
};

// LAYOUT 0: token order to token order; 1: token order to sorted [H, N, D]; 2: sorted to token order.
// A block takes `tokens` rows of `heads_each` heads.  WHOLE: pairs lie within a chunk of 16 bytes, or are the same places of two chunks.
// MAPS: a head is two maps of whole chunks.
template <typename T, bool INTERLEAVED, bool WHOLE, int LAYOUT, bool MAPS>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  constexpr int V = Chunk<T>::V;
  extern __shared__ floatx2_t turn[];   // [tokens][pairs]: cosine, sine, times the factor
  const int half = a.R / 2, chunks = a.D / V;
  const int64_t row0 = (int64_t)blockIdx.x * a.tokens;
  const int rows = (int)min((int64_t)a.tokens, a.N - row0);
  const int angles = MAPS ? a.pairs : half;
  for (int i = threadIdx.x; i < rows * angles; i += 256) {
    const int r = i / angles, p = i - r * angles;
    const int64_t tok = LAYOUT == 0 ? row0 + r : a.perm[row0 + r];
    int axis = 0;
#pragma unroll
    for (int x = 0; x + 1 < kMaxAxes; ++x) axis += x + 1 < a.axes && p >= a.bound[x];
    const double turns = (double)a.pos[axis * a.N + tok] * (a.inv_freq[p] * 0.15915494309189535);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[i] = floatx2_t{c * a.factor, s * a.factor * a.sign};
  }
  __syncthreads();

  const int h0 = blockIdx.y * a.heads_each, nh = min(a.heads_each, a.first[3] - h0);
  // A lane a chunk: (row, head, chunk) of a thread's pieces of work, 256 apart, by carries: a division each would cost as much as the rest.
  // Heads of a token lie beside each other in token order, rows of a head in sorted order: the side that is written is walked.
  const int pairs = half / V, inner = LAYOUT == 1 ? rows : nh;
  int chunk = threadIdx.x % chunks, in = threadIdx.x / chunks % inner, out = threadIdx.x / chunks / inner;
  const int chunk_step = 256 % chunks, in_step = 256 / chunks % inner, out_step = 256 / chunks / inner;
  for (int i = threadIdx.x; i < rows * nh * chunks; i += 256) {
    const int r = LAYOUT == 1 ? in : out, hh = h0 + (LAYOUT == 1 ? out : in);
    const int at = chunk;
    const bool second = MAPS && at >= chunks / 2;
    const int own = second ? at - chunks / 2 : at;   // of its head or map
    chunk += chunk_step;
    in += in_step;
    out += out_step;
    if (chunk >= chunks) chunk -= chunks, ++in;
    if (in >= inner) in -= inner, ++out;
    const int which = (hh >= a.first[1]) + (hh >= a.first[2]);
    const int head = hh - a.first[which], H = a.heads[which];
    const int64_t slot = row0 + r, tok = LAYOUT == 0 ? slot : a.perm[slot];
    const int64_t in_tokens = (tok * H + head) * a.D, in_sorted = ((int64_t)head * a.N + slot) * a.D;
    const T* __restrict__ src = (const T*)a.src[which] + (LAYOUT == 2 ? in_sorted : in_tokens);
    T* __restrict__ dst = (T*)a.dst[which] + (LAYOUT == 1 ? in_sorted : in_tokens);
    const floatx2_t* t = turn + r * angles + (second ? a.second : 0);
    const uintx4_t w = *(const uintx4_t*)(src + at * V);
    if (which == 2 || own * V >= a.R) {
      *(uintx4_t*)(dst + at * V) = w;
      continue;
    }
    float f[V], y[V];
    Chunk<T>::get(w, f);
    if constexpr (INTERLEAVED) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const int p = (own * V + e) / 2;
        if (p < half) {
          const floatx2_t cs = t[p];
          y[e] = f[e] * cs[0] - f[e + 1] * cs[1];
          y[e + 1] = f[e + 1] * cs[0] + f[e] * cs[1];
        } else {
          y[e] = f[e];
          y[e + 1] = f[e + 1];
        }
      }
    } else if constexpr (WHOLE) {
      const bool low = own < pairs;
      const int c = low ? own : own - pairs;
      float o[V];   // the partners, which their own lane loads too: the second read is from L1
      Chunk<T>::get(*(const uintx4_t*)(src + (low ? at + pairs : at - pairs) * V), o);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const floatx2_t cs = t[c * V + e];
        y[e] = f[e] * cs[0] + o[e] * (low ? -cs[1] : cs[1]);
      }
    } else {   // partners anywhere: read one by one
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int d = own * V + e;
        if (d < a.R) {
          const bool low = d < half;
          const floatx2_t cs = t[low ? d : d - half];
          const float other = value(src[at * V + e + (low ? half : -half)]);
          y[e] = low ? f[e] * cs[0] - other * cs[1] : f[e] * cs[0] + other * cs[1];
        } else {
          y[e] = f[e];
        }
      }
    }
    *(uintx4_t*)(dst + at * V) = Chunk<T>::put(y);
  }
}

struct RotaryShape {
  int64_t N;
  int D, axes, R, interleaved, dtype;
  const int* axis_pairs;
  float factor;
  int maps = 1, each = 0;   // maps of a head; each: with pairs of its own
  int pairs() const { return R / 2 * (each ? maps : 1); }
};

int check_rotary(const RotaryShape& s) {
  if (s.N < 0 || s.D < 1 || s.axes < 1 || s.R < 2 || s.R % 2 || s.R > s.D / s.maps) return MOGA_ERR_INVALID_ARG;
  if (!(std::fabs(s.factor) < INFINITY)) return MOGA_ERR_INVALID_ARG;
  if (s.dtype != MOGA_F32 && s.dtype != MOGA_BF16) return MOGA_ERR_UNSUPPORTED;
  if (s.D % (8 * s.maps) || s.D > kMaxHeadDim || s.axes > kMaxAxes || s.N >= ((int64_t)1 << 28)) return MOGA_ERR_UNSUPPORTED;
  if (!s.axis_pairs) return s.axes == 1 ? MOGA_OK : MOGA_ERR_INVALID_ARG;
  int64_t sum = 0;
  for (int a = 0; a < s.axes; ++a) {
    if (s.axis_pairs[a] < 0) return MOGA_ERR_INVALID_ARG;
    sum += s.axis_pairs[a];
  }
  return sum == s.pairs() ? MOGA_OK : MOGA_ERR_INVALID_ARG;
}

template <typename T, int LAYOUT, bool MAPS>
int launch_rotary(RotaryArgs& a, const RotaryShape& s, hipStream_t st) {
  constexpr int V = Chunk<T>::V;
  const int heads = a.first[3], chunks = s.D / V;
  // About 1,024 chunks a block: tokens of one block share nothing but the launch, heads share the angles.  Fewer heads a block where the
  // tokens alone do not fill the chip.  Into sorted order at least four rows, so that a head's writes are 1 KB.
  a.tokens = std::max(LAYOUT == 0 ? 1 : 4, std::min(16, 1024 / std::max(1, heads * chunks)));
  if (a.tokens > s.N) a.tokens = (int)s.N;
  const int64_t row_blocks = (s.N + a.tokens - 1) / a.tokens;
  int parts = (int)std::max<int64_t>(1, std::min<int64_t>(512 / row_blocks, (heads * chunks * a.tokens + 255) / 256));
  a.heads_each = (heads + parts - 1) / parts;
  const dim3 grid((unsigned)row_blocks, (unsigned)((heads + a.heads_each - 1) / a.heads_each));
  if (!grid_fits(row_blocks * grid.y, 256)) return MOGA_ERR_UNSUPPORTED;
  const size_t lds = (size_t)a.tokens * a.pairs * sizeof(floatx2_t);
  if (s.interleaved) rotary_kernel<T, true, true, LAYOUT, MAPS><<<grid, 256, lds, st>>>(a);
  else if (s.R / 2 % V == 0) rotary_kernel<T, false, true, LAYOUT, MAPS><<<grid, 256, lds, st>>>(a);
  else rotary_kernel<T, false, false, LAYOUT, MAPS><<<grid, 256, lds, st>>>(a);
  return launch_status();
}

int rotary(const void* const (&src)[3], void* const (&dst)[3], const int (&heads)[3], const int32_t* perm, int layout, const int32_t* pos,
           const double* inv_freq, const RotaryShape& s, float sign, hipStream_t st) {
  const int bad = check_rotary(s);
  if (bad) return bad;
  RotaryArgs a = {};
  int total = 0;
  for (int i = 0; i < 3; ++i) {
    if (heads[i] < 0 || heads[i] > 65536) return heads[i] < 0 ? MOGA_ERR_INVALID_ARG : MOGA_ERR_UNSUPPORTED;
    a.first[i] = total;
    total += heads[i];
    a.heads[i] = heads[i];
    a.src[i] = src[i];
    a.dst[i] = dst[i];
  }
  a.first[3] = total;
  if (total < 1) return MOGA_ERR_INVALID_ARG;
  if (s.N == 0) return MOGA_OK;
  if (!pos || !inv_freq || (layout && !perm)) return MOGA_ERR_INVALID_ARG;
  if (!aligned16(pos) || !aligned16(inv_freq)) return MOGA_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (heads[i] && (!src[i] || !dst[i] || !aligned16(src[i]) || !aligned16(dst[i]) || src[i] == dst[i])) return MOGA_ERR_INVALID_ARG;
  a.pos = pos;
  a.inv_freq = inv_freq;
  a.perm = perm;
  a.N = s.N;
  a.D = s.D;
  a.R = s.R;
  a.axes = s.axes;
  a.pairs = s.pairs();
  a.second = s.each ? s.R / 2 : 0;
  for (int x = 0, n = 0; x < kMaxAxes; ++x) a.bound[x] = n += !s.axis_pairs ? (x == 0 ? a.pairs : 0) : x < s.axes ? s.axis_pairs[x] : 0;
  a.factor = s.factor;
  a.sign = sign;
#define MOGA_ROTARY(T)                                                                                                              \
  (s.maps == 2   ? layout == 1 ? launch_rotary<T, 1, true>(a, s, st) : launch_rotary<T, 2, true>(a, s, st)                          \
   : layout == 0 ? launch_rotary<T, 0, false>(a, s, st)                                                                             \
   : layout == 1 ? launch_rotary<T, 1, false>(a, s, st) : launch_rotary<T, 2, false>(a, s, st))
  return s.dtype == MOGA_F32 ? MOGA_ROTARY(float) : MOGA_ROTARY(unsigned short);
#undef MOGA_ROTARY
}

}  // namespace
}  // namespace moga

using namespace moga;

extern "C" int moga_rotary_fwd(const void* q, const void* k, int dtype, int64_t N, int Hq, int Hk, int D, const int32_t* positions, int axes,
                               const int* axis_pairs, const double* inv_freq, int R, int interleaved, float factor, void* qo, void* ko,
                               void* stream) {
  return rotary({q, k, nullptr}, {qo, ko, nullptr}, {Hq, Hk, 0}, nullptr, 0, positions, inv_freq,
                {N, D, axes, R, interleaved, dtype, axis_pairs, factor}, 1.f, (hipStream_t)stream);
}

extern "C" int moga_rotary_bwd(const void* d_qo, const void* d_ko, int dtype, int64_t N, int Hq, int Hk, int D, const int32_t* positions,
                               int axes, const int* axis_pairs, const double* inv_freq, int R, int interleaved, float factor, void* d_q,
                               void* d_k, void* stream) {
  return rotary({d_qo, d_ko, nullptr}, {d_q, d_k, nullptr}, {Hq, Hk, 0}, nullptr, 0, positions, inv_freq,
                {N, D, axes, R, interleaved, dtype, axis_pairs, factor}, -1.f, (hipStream_t)stream);
}

extern "C" int moga_rotary_permute_fwd(const void* q, const void* k, const void* v, int dtype, int64_t N, int H, int D, const int32_t* perm,
                                       const int32_t* positions, int axes, const int* axis_pairs, const double* inv_freq, int R,
                                       int interleaved, float factor, void* qh, void* kh, void* vh, void* stream) {
  if (H < 1) return MOGA_ERR_INVALID_ARG;
  return rotary({q, k, v}, {qh, kh, vh}, {H, H, H}, perm, 1, positions, inv_freq, {N, D, axes, R, interleaved, dtype, axis_pairs, factor}, 1.f,
                (hipStream_t)stream);
}

extern "C" int moga_rotary_permute_bwd(const void* d_qh, const void* d_kh, const void* d_vh, int dtype, int64_t N, int H, int D,
                                       const int32_t* perm, const int32_t* positions, int axes, const int* axis_pairs, const double* inv_freq,
                                       int R, int interleaved, float factor, void* d_q, void* d_k, void* d_v, void* stream) {
  if (H < 1) return MOGA_ERR_INVALID_ARG;
  return rotary({d_qh, d_kh, d_vh}, {d_q, d_k, d_v}, {H, H, H}, perm, 2, positions, inv_freq,
                {N, D, axes, R, interleaved, dtype, axis_pairs, factor}, -1.f, (hipStream_t)stream);
}

extern "C" int moga_rotary_permute_maps_fwd(const void* q, const void* k, const void* v, int dtype, int64_t N, int H, int D, const int32_t* perm,
                                            const int32_t* positions, int axes, const int* axis_pairs, const double* inv_freq, int R, int each_map,
                                            int interleaved, float factor, void* qh, void* kh, void* vh, void* stream) {
  if (H < 1) return MOGA_ERR_INVALID_ARG;
  return rotary({q, k, v}, {qh, kh, vh}, {H, H, H}, perm, 1, positions, inv_freq,
                {N, D, axes, R, interleaved, dtype, axis_pairs, factor, 2, each_map}, 1.f, (hipStream_t)stream);
}

extern "C" int moga_rotary_permute_maps_bwd(const void* d_qh, const void* d_kh, const void* d_vh, int dtype, int64_t N, int H, int D,
                                            const int32_t* perm, const int32_t* positions, int axes, const int* axis_pairs, const double* inv_freq,
                                            int R, int each_map, int interleaved, float factor, void* d_q, void* d_k, void* d_v, void* stream) {
  if (H < 1) return MOGA_ERR_INVALID_ARG;
  return rotary({d_qh, d_kh, d_vh}, {d_q, d_k, d_v}, {H, H, H}, perm, 2, positions, inv_freq,
                {N, D, axes, R, interleaved, dtype, axis_pairs, factor, 2, each_map}, -1.f, (hipStream_t)stream);
}

// Host only.  All in 64 bits.
extern "C" int moga_rotary_build_freqs(int R, double base, int scaling, double scale_factor, double original_len, double beta_fast,
                                       double beta_slow, double* inv_freq, float* factor) {
  if (R < 0 || R % 2 || !inv_freq || !factor || !(base > 0.) || !std::isfinite(base)) return MOGA_ERR_INVALID_ARG;
  if (scaling < MOGA_ROTARY_PLAIN || scaling > MOGA_ROTARY_PARTS) return MOGA_ERR_UNSUPPORTED;
  if (scaling != MOGA_ROTARY_PLAIN && (!(scale_factor >= 1.) || !std::isfinite(scale_factor))) return MOGA_ERR_INVALID_ARG;
  if (scaling == MOGA_ROTARY_PARTS &&
      (!(original_len > 0.) || !std::isfinite(original_len) || !(beta_slow > 0.) || !(beta_fast > beta_slow) || !std::isfinite(beta_fast)))
    return MOGA_ERR_INVALID_ARG;
  const int n = R / 2;
  if (scaling == MOGA_ROTARY_BASE && n > 1) base *= std::pow(scale_factor, (double)n / (n - 1));
  for (int i = 0; i < n; ++i) {
    double f = std::pow(base, -(double)i / n);
    if (scaling == MOGA_ROTARY_LINEAR) f /= scale_factor;
    if (scaling == MOGA_ROTARY_PARTS) {
      const double turns = original_len * f / 6.283185307179586;
      const double keep = std::min(1., std::max(0., (turns - beta_slow) / (beta_fast - beta_slow)));
      f = keep * f + (1. - keep) * f / scale_factor;
    }
    inv_freq[i] = f;
  }
  *factor = scaling == MOGA_ROTARY_PARTS ? (float)(0.1 * std::log(scale_factor) + 1.) : 1.f;
  return MOGA_OK;
}
