// Differential attention inside groups: pieces that its forward and backward kernels share.
//
// A head's D channels of Q and K are two halves, a map each:  A_m = softmax(s Q_m K_m^T), m = 1, 2, over the keys of the query's group;
//   O = A_1 V - lambda_h A_2 V.
// Everything is computed by 16-row matrix products whose fragments hold eight consecutive channels or rows per lane, in either type: a bf16
// fragment is one operand of a 16x16x32 product, an fp32 one eight operands of 16x16x4 products (lane group g's element j stands for channel
// 8 g + j in both).  Scores come out transposed to what the next product reads, so that weights never leave their lanes (attn_common.h).
#pragma once

#include "attn_pipe.h"

namespace moga {

struct FragF32 {
  floatx4_t lo, hi;
  __device__ __forceinline__ float at(int i) const { return i < 4 ? lo[i] : hi[i - 4]; }
};
template <typename T> struct FragOf { typedef bf16x8_t type; };
template <> struct FragOf<float> { typedef FragF32 type; };
template <typename T> using Frag = typename FragOf<T>::type;

__device__ __forceinline__ floatx4_t mma(const bf16x8_t& a, const bf16x8_t& b, const floatx4_t& c) { return mfma16(a, b, c); }
__device__ __forceinline__ floatx4_t mma(const FragF32& a, const FragF32& b, floatx4_t c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.at(i), b.at(i), c, 0, 0, 0);
  return c;
}
// Eight weights as an operand; bf16: to nearest even, what the matrix instruction takes.
__device__ __forceinline__ void make_frag(bf16x8_t& f, const float (&v)[8]) {
  f = __builtin_bit_cast(bf16x8_t, uintx4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
}
__device__ __forceinline__ void make_frag(FragF32& f, const float (&v)[8]) {
  f.lo = floatx4_t{v[0], v[1], v[2], v[3]};
  f.hi = floatx4_t{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void load_frag(bf16x8_t& f, const unsigned short* p) { f = *(const bf16x8_t*)p; }
__device__ __forceinline__ void load_frag(FragF32& f, const float* p) {
  f.lo = *(const floatx4_t*)p;
  f.hi = *(const floatx4_t*)(p + 4);
}

// Fragments of a wave's 16 NC rows from row0 (clamped to the last row of the group): columns 16 c + r, channels 32 kb + 8 g ..
template <typename T, int D, int NC>
__device__ __forceinline__ void diff_columns(Frag<T> (&f)[NC][D / 32], const T* __restrict__ src, int row0, int ge, int64_t head_off) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const T* p = src + (head_off + min(row0 + 16 * c + (lane & 15), ge - 1)) * D + 8 * (lane >> 4);
#pragma unroll
    for (int kb = 0; kb < D / 32; ++kb) load_frag(f[c][kb], p + 32 * kb);
  }
}

// Rows of a group streamed through LDS, 32 of two tensors at a time.  ready(s): tile s may be read, by all waves of the block together, and
// all of them have left tile s - KEEP.
// nat(which, t, kb): operand t of the tile's rows (step_row), channels 32 kb ..; tr(which, dt): transposed, channels 16 dt .., all 32 rows.
template <typename T, int D, bool ROWS = false, int KEEP = 1, int SLOTS = 4> struct DiffTiles;

// With ROWS, four constants of every row beside them: rows(v, i), constant v of rows i .. i + 3.
// bf16: direct-to-LDS loads into a ring of SLOTS, as far ahead as the tiles that are kept allow.
template <bool ROWS, int KEEP, int SLOTS> struct DiffTiles<unsigned short, 128, ROWS, KEEP, SLOTS> {
  static constexpr int kSlots = SLOTS, kTile = 32 * kHeadDim * 2, kLoads = 2 * kDmaLoads<4, 32> + ROWS, kAhead = SLOTS - KEEP, kRowSlot = 640;
  struct Lds {
    __attribute__((aligned(1024))) unsigned short a[SLOTS][32 * kHeadDim];
    __attribute__((aligned(1024))) unsigned short b[SLOTS][32 * kHeadDim];
    __attribute__((aligned(128))) char rows[ROWS ? SLOTS : 1][ROWS ? kRowSlot : 16];
  };
  PipeDma dma;
  unsigned n_[2], t_[2][2], off, rows_lds, rows_own, rows_at;
  const void* rows_base;
  // Wave v moves constant v of the 32 rows, and v + 1 (the same bytes twice) with the lanes that are left.  Each constant by itself: the four
  // rows that a lane group wants are one read, and the four lane groups' reads lie in different banks (as 16 bytes a row they do not,
  // and a read takes 50 cycles).
  __device__ __forceinline__ void issue(int s) {
    pipe_issue<4, 32, false>(dma, 32 * s, (s & (SLOTS - 1)) * kTile);
    if constexpr (ROWS) {
      const int lane = threadIdx.x & 63, v = min((int)(threadIdx.x >> 6) + (lane >> 5), 3), row = min(32 * s + (lane & 31), dma.last_row);
      lds_dma4_soff(rows_base, (unsigned)row * 16u + v * 4u, rows_own + (s & (SLOTS - 1)) * kRowSlot);
    }
  }
  __device__ __forceinline__ void start(Lds& lds, const unsigned short* a, const unsigned short* b, int n, const floatx4_t* rows = nullptr) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    dma.kbase = uniform_ptr(a);
    dma.vbase = uniform_ptr(b);
    dma_lanes<4, 32>(dma, &lds.a[0][0], &lds.b[0][0], wave, lane);
    dma.last_row = n - 1;
    if constexpr (ROWS) {
      rows_base = uniform_ptr(rows);
      rows_lds = lds_addr_uniform(&lds.rows[0][0]);
      rows_own = rows_lds + wave * 128;
    }
    n_[0] = nat_address(&lds.a[0][0], lane);
    n_[1] = nat_address(&lds.b[0][0], lane);
    tr_addresses(t_[0], &lds.a[0][0], lane);
    tr_addresses(t_[1], &lds.b[0][0], lane);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) issue(s);   // rows are clamped: always issued
  }
  __device__ __forceinline__ void ready(int s) {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(kLoads * (kAhead - 1)));
    // tile s is here, and every wave has left tile s - KEEP, whose slot is filled again (kept for longer, a wave's reads of it are done)
    if constexpr (KEEP == 1) __syncthreads();
    else block_barrier();
    issue(s + kAhead);
    at(s);
  }
  __device__ __forceinline__ void at(int s) {   // nat, tr and row read tile s from here on
    off = (unsigned)(s & (SLOTS - 1)) * kTile;
    if constexpr (ROWS) rows_at = rows_lds + (unsigned)(s & (SLOTS - 1)) * kRowSlot;
  }
  __device__ __forceinline__ void finish() { __builtin_amdgcn_s_waitcnt(waitcnt_vm(0)); }   // before the LDS is released
  __device__ __forceinline__ bf16x8_t nat(int which, int t, int kb) const { return read_nat<32>(n_[which] + off, t, kb); }
  __device__ __forceinline__ bf16x8_t tr(int which, int dt) const { return read_tr<32>(t_[which], off, dt); }
  __device__ __forceinline__ floatx4_t rows(int v, int i) const {
    return *(const floatx4_t __attribute__((address_space(3)))*)(uintptr_t)(rows_at + 128 * v + 4 * i);
  }
};

// The same for a wave by itself: every fourth tile of the block's, a ring of two, no barriers.
struct DiffWaveTiles {
  static constexpr int kTile = 32 * kHeadDim * 2, kLoads = 2 * kDmaLoads<1, 32>;
  struct Lds {
    __attribute__((aligned(1024))) unsigned short a[2][32 * kHeadDim];
    __attribute__((aligned(1024))) unsigned short b[2][32 * kHeadDim];
  };
  PipeDma dma;
  unsigned n_[2], t_[2][2], off;
  __device__ __forceinline__ void start(Lds& lds, const unsigned short* a, const unsigned short* b, int n, int first) {
    const int lane = threadIdx.x & 63;
    dma.kbase = uniform_ptr(a);
    dma.vbase = uniform_ptr(b);
    dma_lanes<1, 32>(dma, &lds.a[0][0], &lds.b[0][0], 0, lane);
    dma.last_row = n - 1;
    n_[0] = nat_address(&lds.a[0][0], lane);
    n_[1] = nat_address(&lds.b[0][0], lane);
    tr_addresses(t_[0], &lds.a[0][0], lane);
    tr_addresses(t_[1], &lds.b[0][0], lane);
    off = kTile;
    issue(first, 0);
    issue(first + 4, kTile);
  }
  __device__ __forceinline__ void issue(int tile, unsigned slot) {   // rows are clamped: always issued
    // 16 rows (1 KB of LDS of each quarter) at a time
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = 16 * h + (int)((threadIdx.x & 63) >> 2);
      const unsigned at = (unsigned)min(32 * tile + row, dma.last_row) * (kHeadDim * 2) + ((((threadIdx.x & 3) ^ lds_swizzle(row))) << 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lds_dma16_soff(dma.kbase, at + 64 * i, dma.lds_k + slot + h * 1024 + i * kQuarterBytes<32>);
        lds_dma16_soff(dma.vbase, at + 64 * i, dma.lds_v + slot + h * 1024 + i * kQuarterBytes<32>);
      }
    }
  }
  __device__ __forceinline__ void next() {   // the next of the wave's tiles may be read
    off ^= kTile;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(kLoads));
    asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ void refill(int tile) {   // its slot is read no more
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    issue(tile, off);
  }
  __device__ __forceinline__ void finish() { __builtin_amdgcn_s_waitcnt(waitcnt_vm(0)); }
  __device__ __forceinline__ bf16x8_t nat(int which, int t, int kb) const { return read_nat<32>(n_[which] + off, t, kb); }
  __device__ __forceinline__ bf16x8_t tr(int which, int dt) const { return read_tr<32>(t_[which], off, dt); }
};

// fp32: through registers, one tile ahead.
template <int D, bool ROWS> struct DiffTiles<float, D, ROWS, 1, 4> {
  static constexpr int kPitch = D + 4, kEach = 32 * D / 4 / 256;
  struct Lds {
    float a[32][kPitch], b[32][kPitch];
    float rows[ROWS ? 4 : 1][32];
  };
  Lds* lds;
  const float *pa, *pb;
  int last;
  floatx4_t ra[kEach], rb[kEach];
  float rr;
  const floatx4_t* constants;
  __device__ __forceinline__ void fetch(int s) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = threadIdx.x + 256 * i, col = e % (D / 4) * 4;
      const int64_t row = min(32 * s + e / (D / 4), last);
      ra[i] = *(const floatx4_t*)(pa + row * D + col);
      rb[i] = *(const floatx4_t*)(pb + row * D + col);
    }
    if (ROWS && threadIdx.x < 128) rr = ((const float*)(constants + min(32 * s + (int)(threadIdx.x & 31), last)))[threadIdx.x >> 5];
  }
  __device__ __forceinline__ void start(Lds& l, const float* a, const float* b, int n, const floatx4_t* r = nullptr) {
    lds = &l;
    constants = r;
    pa = a;
    pb = b;
    last = n - 1;
    fetch(0);
  }
  __device__ __forceinline__ void ready(int s) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = threadIdx.x + 256 * i, row = e / (D / 4), col = e % (D / 4) * 4;
      *(floatx4_t*)&lds->a[row][col] = ra[i];
      *(floatx4_t*)&lds->b[row][col] = rb[i];
    }
    if (ROWS && threadIdx.x < 128) lds->rows[threadIdx.x >> 5][threadIdx.x & 31] = rr;
    __syncthreads();
    fetch(s + 1);
  }
  __device__ __forceinline__ void finish() {}
  __device__ __forceinline__ floatx4_t rows(int v, int i) const { return *(const floatx4_t*)&lds->rows[v][i]; }
  __device__ __forceinline__ FragF32 nat(int which, int t, int kb) const {
    const int lane = threadIdx.x & 63;
    const float* p = (which ? lds->b : lds->a)[step_row(lane & 15) + 4 * t] + 32 * kb + 8 * (lane >> 4);
    FragF32 f;
    load_frag(f, p);
    return f;
  }
  __device__ __forceinline__ FragF32 tr(int which, int dt) const {
    const int lane = threadIdx.x & 63;
    const float(*p)[kPitch] = (which ? lds->b : lds->a) + 8 * (lane >> 4);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i][16 * dt + (lane & 15)];
    FragF32 f;
    make_frag(f, v);
    return f;
  }
};

// Four results of column c, d tiles dt (channels 16 dt + 4 g ..), at `row`.
__device__ __forceinline__ void store4(float* row, int dt, const floatx4_t& v) { *(floatx4_t*)(row + 16 * dt + 4 * ((threadIdx.x & 63) >> 4)) = v; }
__device__ __forceinline__ void store4(unsigned short* row, int dt, const floatx4_t& v) {
  *(uintx2_t*)(row + 16 * dt + 4 * ((threadIdx.x & 63) >> 4)) = pack4(v, 1.f);
}

}  // namespace moga
