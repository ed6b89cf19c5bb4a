// Tiles of matrix products C[M][N] = sum_k A(m, k) B(n, k), the operands as they lie in memory.
//
// A block owns BM x BN of C and walks K in steps of 128 bytes of an operand's row (64 bf16, 32 fp32).  Either operand lies with k last ("rows":
// an activation, or a weight as it is) or with k first ("columns": the same tensor as the operand of its gradient, without a transposed copy).
// Both are staged global -> LDS by direct loads, 16 bytes a lane, two steps in turn, and read back as MFMA operands: rows with 16-byte
// reads, bf16 columns with transposed 8-byte reads, fp32 columns with 4-byte reads.  Chunks of a staged row are exchanged (xor) so that the lanes of
// a read fall on different banks; the exchange is made in the global addresses, since a direct load fills LDS in lane order.
// Rows, columns and k past the operand's end are read as zeros: their buffer offset is put past the buffer's range.
// Direct loads need no registers on the way and leave the vector units free: the address of a load is one of a thread's few offsets plus a scalar base
// that moves on by a step.  Steps of 128 bytes are whole lines of either layout.
#pragma once

#include "lds_pipe.h"

namespace moga {

constexpr unsigned kBufferBytes = 0x7ffffff0u, kPastBuffer = 0x80000000u;

// 16 bytes a lane from `base + voff` to LDS (the wave's 1 KB at lds_wave_base); zeros where voff is kPastBuffer.  base and lds_wave_base are
// wave-uniform and in scalar registers.
__device__ __forceinline__ void lds_dma16_buffer(uint64_t base, unsigned voff, unsigned lds_wave_base) {
  const uintx4_t rsrc = {(unsigned)base, (unsigned)(base >> 32), kBufferBytes, 0x00020000u};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds_wave_base), "v"(voff), "s"(rsrc) : "memory");
}
__device__ __forceinline__ uint64_t uniform_address(const void* p) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  return (unsigned)__builtin_amdgcn_readfirstlane((unsigned)a) | (uint64_t)((unsigned)__builtin_amdgcn_readfirstlane((unsigned)(a >> 32)) & 0xffffu) << 32;
}

// All waves of the block are here.  Unlike __syncthreads it does not wait for the wave's own LDS reads.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <typename T> struct Frag;
template <> struct Frag<unsigned short> { bf16x8_t v; };
template <> struct Frag<float> { floatx4_t v; };

__device__ __forceinline__ void mfma_frag(floatx4_t& c, Frag<unsigned short> a, Frag<unsigned short> b) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
// k = 4 g + j of lane group g in product j, in both operands
__device__ __forceinline__ void mfma_frag(floatx4_t& c, Frag<float> a, Frag<float> b) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
}

// One operand of a block: ROWS rows (or columns) by 128 bytes of k a step, staged by the block; a wave reads TILES tiles of 16 from tile `first` on,
// in two halves of k.
template <typename T, bool KFIRST, int ROWS, int THREADS, int TILES>
struct Operand {
  static constexpr int ES = sizeof(T), V = 16 / ES, BK = 128 / ES, L = ROWS * 8 / THREADS, CPR = ROWS * ES / 16;
  static constexpr unsigned kBytes = ROWS * 128;
  static_assert(ROWS == 64 || ROWS == 128 || ROWS == 256);   // exchanges stay within a row
  uint64_t base;     // address of this block's rows at the k of the next step to be staged
  uint64_t base2;    // of the second half of the rows of each 64 (init_paired)
  int64_t step_bytes;
  unsigned lds_to;   // of the wave's first load of that step
  unsigned voff[L];
  int kofs[KFIRST ? L : 1];
  unsigned read[KFIRST ? TILES : 2];   // lane's LDS addresses
  int k_left;                          // from the next step to be staged on

  __device__ __forceinline__ static int swizzle(int k) {   // columns: exchanged 16-byte chunks of row k
    // a read's half wave touches, bf16, k 0 .. 3 and 8 .. 11 by 32 bytes, of rows of 128 bytes two beside each other; fp32, k 0, 4, 8, 12 by 64
    if (ES == 4) return ((k >> 2) & 3) * 4;
    return ROWS == 64 ? (((k >> 1) & 1) | ((k >> 2) & 2)) * 2 : ((k & 3) | ((k >> 1) & 4)) * 2;
  }
  __device__ __forceinline__ static int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

  // rows r0 .. of a matrix [R][ld], or columns r0 .. of a matrix [..][ld]; k_count of k from k0 on
  __device__ __forceinline__ void init(const T* p, int64_t ld, int64_t r0, int64_t R, int64_t k0, int k_count, int first, unsigned lds) {
    k_left = k_count;
    base = uniform_address(KFIRST ? p + k0 * ld + r0 : p + r0 * ld + k0);
    step_bytes = KFIRST ? (int64_t)BK * ld * ES : 128;
    const int64_t left = R - r0;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int q = i * THREADS + threadIdx.x;
      if constexpr (KFIRST) {
        const int k = q / CPR, c = (q % CPR) ^ swizzle(k);
        kofs[i] = k;
        voff[i] = c * V < left ? (unsigned)(k * ld * ES + c * 16) : kPastBuffer;
      } else {
        const int j = q >> 3, c = (q & 7) ^ ((j >> 1) & 7);
        kofs[0] = c * V;   // the same in every i
        voff[i] = j < left ? (unsigned)(j * ld * ES + c * 16) : kPastBuffer;
      }
    }
    init_read(first, lds);
  }
  // Of each 64 staged rows 32 are rows f0 + .. of a matrix [2 F][ld] and 32 the same rows of its second half.
  __device__ __forceinline__ void init_paired(const T* p, int64_t ld, int64_t f0, int64_t F, int k_count, int first, unsigned lds) {
    static_assert(!KFIRST && (THREADS == 256 || THREADS == 512));
    k_left = k_count;
    base = uniform_address(p + f0 * ld);
    base2 = base + F * ld * ES;
    if (THREADS == 512 && (wave() & 4)) base = base2;   // the upper waves of a block of eight load them, the odd loads of a block of four
    step_bytes = 128;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int q = i * THREADS + threadIdx.x, j = q >> 3, c = (q & 7) ^ ((j >> 1) & 7), f = (j >> 6) * 32 + (j & 31);
      kofs[0] = c * V;
      voff[i] = f < F - f0 ? (unsigned)(f * ld * ES + c * 16) : kPastBuffer;
    }
    init_read(first, lds);
  }
  __device__ __forceinline__ void init_read(int first, unsigned lds) {
    lds_to = lds + wave() * 1024;
    const int l = threadIdx.x & 63, r = l & 15, g = l >> 4;
    if constexpr (!KFIRST) {
#pragma unroll
      for (int h = 0; h < 2; ++h) read[h] = lds + (first * 16 + r) * 128 + (((h * 4 + g) ^ (r >> 1)) & 7) * 16;
    } else {
      const int k = ES == 2 ? 8 * g + (r >> 2) : 4 * g;
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const int col = (first + j) * 16 + (ES == 2 ? (r & 3) * 4 : r), c = (col / V) ^ swizzle(k);
        read[j] = lds + k * ROWS * ES + c * 16 + col % V * ES;
      }
    }
  }

  // The i-th of the thread's loads of the next step
  template <bool PAIRED = false>
  __device__ __forceinline__ void stage(int i) const {
    lds_dma16_buffer(PAIRED && THREADS == 256 && (i & 1) ? base2 : base, kofs[KFIRST ? i : 0] < k_left ? voff[i] : kPastBuffer,
                     lds_to + i * THREADS * 16);
  }
  // On to the step after it, whose buffer lies `other` bytes on
  template <bool PAIRED = false>
  __device__ __forceinline__ void advance(int other) {
    base += step_bytes;
    if (PAIRED) base2 += step_bytes;
    k_left -= BK;
    lds_to += other;
  }
  // Reads of half h go to the other buffer (columns: those of both halves, with half 0)
  __device__ __forceinline__ void turn(int h, int other) {
    if constexpr (!KFIRST) {
      read[h] += other;
    } else if (h == 0) {
#pragma unroll
      for (int j = 0; j < TILES; ++j) read[j] += other;
    }
  }
  // Operand of the wave's tile, half h of the step
  __device__ __forceinline__ Frag<T> get(int tile, int h) const {
    Frag<T> f;
    if constexpr (!KFIRST) {
      f.v = __builtin_bit_cast(decltype(f.v), *(const uintx4_t __attribute__((address_space(3)))*)(uintptr_t)(read[h] + tile * 2048));
    } else if constexpr (ES == 2) {
      const unsigned at = read[tile] + h * 32 * ROWS * 2;
      f.v = concat_tr(lds_read_tr16_addr(at), lds_read_tr16_addr(at + 4 * ROWS * 2));
    } else {
      const unsigned at = read[tile] + h * 16 * ROWS * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = *(const float __attribute__((address_space(3)))*)(uintptr_t)(at + j * ROWS * 4);
    }
    return f;
  }
};

// Which tile block b takes.  Blocks go to the eight XCDs in turn, and 256 of them run at a time: those are a square of about 16 x 16 tiles, whose
// operands pass the cache that the XCDs share once, and the 32 of an XCD are 8 x 4 tiles of it, whose operands pass its own.
__device__ __forceinline__ void tile_of(unsigned b, unsigned tiles_m, unsigned tiles_n, unsigned& bm, unsigned& bn) {
  const unsigned tiles = tiles_m * tiles_n, whole = tiles & ~255u;
  unsigned at;
  if (b < whole) {
    at = (b & ~255u) + (b & 7) * 32 + ((b >> 3) & 31);
  } else {   // eighths of what is left
    const unsigned left = tiles - whole, x = b & 7, per = left >> 3, more = left & 7;
    at = whole + x * per + min(x, more) + ((b - whole) >> 3);
  }
  // panels of `high` rows of tiles, in them groups of 16 columns, in them strips of 8 rows, down the columns of a strip
  const unsigned high = tiles_n >= 16 ? 16 : max(8u, 256 / tiles_n & ~7u);
  const unsigned panel = at / (high * tiles_n), h = min(high, tiles_m - panel * high);
  at -= panel * high * tiles_n;
  const unsigned group = at / (h * 16), w = min(16u, tiles_n - group * 16);
  at -= group * h * 16;
  const unsigned strip = at / (8 * w), rows = min(8u, h - strip * 8);
  at -= strip * 8 * w;
  bm = panel * high + strip * 8 + at % rows;
  bn = group * 16 + at / rows;
}

}  // namespace moga
