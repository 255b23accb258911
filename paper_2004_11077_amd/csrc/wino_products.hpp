// Matrix products of the training operators (linear cross entropy, orthogonalised updates):
//   D[m][n] = sum_k A(m, k) B(n, k)
// on the matrix pipe (v_mfma_f32_16x16x32_bf16 / _f16, fp32 accumulation).
//
// An operand is NP planes of 16-bit values that add up to its values.  NP = 1: bf16 values as they
// stand.  NP = 2: fp16, x as fp16(x) + fp16(x - fp16(x)), 22 significant bits, and three of the four
// products of two such sums: the one left out is below 2^-22 of the term.  fp16's narrow exponent
// wants x times a power of two, so that the largest magnitude is 2^15 or below (half of what fp16
// holds); what is smaller than 2^-18 of that keeps 2^-40 of it.  Products of two such values are exact
// in fp32, so a sum is as good as one of fp32 products (measured against 64 bits: better, because a
// block of 32 k costs three roundings of the sum and not 32), at three matrix instructions of 2.5
// PFLOP/s instead of one fp32 instruction of 0.157 PFLOP/s.
//
// Tile: BM x BN of D per work group, WM x WN waves, 16 x 16 blocks of D per instruction, for which a
// lane holds eight consecutive k of one row of an operand.  A stage of 32 k of every plane is copied
// from memory straight into LDS (buffer_load ... lds), a lane's 16 bytes behind the lane before's; a
// lane may fetch from anywhere, so the order in LDS is free:
//   * an operand with k along its rows in memory: 16 rows x 32 k are one KiB, lane l's 16 bytes at
//     16 l are what lane l of the instruction takes.  One conflict-free read, no address arithmetic.
//   * an operand with k across the rows (ACROSS): 8 k x 64 m are one KiB, whole lines from memory.
//     ds_read_b64_tr_b16 hands a lane four consecutive k of its m; 16-byte pieces of a row change
//     places by its k (swap_of), so that the rows a read touches lie in different banks.
// No operand is therefore ever transposed in memory.  RING buffers, RING - 1 stages under way: a wave
// waits until its own copies of a stage have landed (counted, so that the later stages' stay under
// way), the barrier then says so of all waves, and also that the buffer of the stage before may be
// filled again.  What lies outside an operand lies outside its buffer descriptor and reads as zeros; k
// runs in whole blocks of 32: along rows the caller pads with zeros.  A work group's first row exists,
// and kMaxLd bounds the offsets within a stage to 31 bits.
// 65536 x 4096 x 2048, bf16 (the plain library product: 1180 TFLOP/s):
//   128 x 128 tiles, 4 waves, two buffers of 64 k, all copies waited for   582 TFLOP/s
//   256 x 256, 8 waves, the same                                            877
//   256 x 256, 8 waves, ring of four, counted waits                         987
//   and the multiplying wave before the fetching one (s_setprio)           1052
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "wino_kernels.hpp"

namespace wino {
namespace prod {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr long kMaxLd = 1L << 21;   // elements between rows: 256 rows of it are 2^30 bytes

// One operand: plane q, batch b, row r, element e at p + q plane + b batch + r ld + e; `rows` rows of
// `cols` elements.  k along the rows: m or n is r, k is e.  ACROSS: k is r, m or n is e.
struct Operand {
  const uint16_t* p;
  long ld, plane, batch;
  int rows, cols;
};

__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ float bf16_value(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
__device__ __forceinline__ uint16_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ __forceinline__ float f16_value(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
__device__ __forceinline__ float power(int e) { return __builtin_ldexpf(1.f, e); }

// x as NP 16-bit values (see above).
template <int NP>
__device__ __forceinline__ void cut(float x, uint16_t (&out)[NP]) {
  if constexpr (NP == 1) {
    out[0] = bf16_bits(x);
  } else {
    out[0] = f16_bits(x);
    out[1] = f16_bits(x - f16_value(out[0]));
  }
}

// One instruction of 16 x 16 x 32.
template <int NP>
__device__ __forceinline__ f32x4 multiply_block(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (NP == 2)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int BM_, int BN_, int WM_, int WN_, int NP_, int RING_, bool AX_ = false, bool BX_ = false>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NP = NP_, RING = RING_;
  static constexpr bool AX = AX_, BX = BX_;                    // k across the rows of A, of B
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 blocks per wave
  static constexpr int RA = BM / 16, RB = BN / 16;             // KiB of a stage's plane of the operands
  static constexpr int STAGE = NP * (RA + RB) * 1024;          // bytes
  static constexpr int LDS = RING * STAGE;
  // copies of a stage per wave and plane; where there are fewer KiB than waves, several waves copy
  // the same one, so that all count alike
  static constexpr int NA = (RA + NW - 1) / NW, NB = (RB + NW - 1) / NW;
  static constexpr int COPIES = NP * (NA + NB);
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && RING >= 2 && LDS <= 160 * 1024);
  static_assert((RA % NW == 0 || NW % RA == 0) && (RB % NW == 0 || NW % RB == 0));
  static_assert((!AX || BM % 64 == 0) && (!BX || BN % 64 == 0));
  static_assert(COPIES * (RING - 2) < 64);   // what a counted wait can say
};

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const uint16_t* p, long bytes) {
  const int size = bytes < 0 ? 0 : bytes > 0x7fffffff ? 0x7fffffff : (int)bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, size, 0x00020000);
}

// Waits until at most N of this wave's copies are under way.  Its LDS reads have all been used by then;
// saying so costs nothing and makes the barrier behind it mean that the buffer is free.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// Places of the 16-byte pieces of a row k of an ACROSS block: piece c lies at c ^ swap_of(k).  A read
// touches rows 8 g + r (+ 4) of four lane groups g, four r each, two neighbouring pieces of a row; rows are
// 128 bytes, so the pair of banks goes by r % 2, and within it the four places by r / 2 and g % 2.
__device__ __forceinline__ int swap_of(int k) { return ((k >> 1) & 1) * 2 + ((k >> 3) & 1) * 4; }

// One operand's side of a tile: SIDE rows (m or n), X: k across.
template <int SIDE, bool X, int NP, int NW>
struct Side {
  static constexpr int R = SIDE / 16, N = (R + NW - 1) / NW;
  const uint16_t* base[NP];
  long bytes, step;          // from the base to the operand's end; ACROSS: elements of a stage
  __amdgpu_buffer_rsrc_t rsrc[NP];
  int at[N];                 // a copy's source, in bytes from the base
  int read[4];               // ACROSS: a lane's place in a stage for the m-blocks 0 .. 3 of 64

  __device__ __forceinline__ Side(const Operand& o, long batch, int first, int k, int lane, int wave) {
    const long start = X ? (long)k * o.ld + first : (long)first * o.ld;
#pragma unroll
    for (int q = 0; q < NP; ++q) base[q] = o.p + q * o.plane + batch * o.batch + start;
    if constexpr (X) {
      bytes = ((long)(o.rows - 1) * o.ld + o.cols - start) * 2;
      step = 32 * o.ld;
    } else {
      int rows = o.rows - first;
      rows = rows < SIDE ? rows : SIDE;
      bytes = ((long)(rows - 1) * o.ld + o.cols) * 2;
      step = 0;
#pragma unroll
      for (int q = 0; q < NP; ++q) rsrc[q] = window(base[q], bytes);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int block = (i * NW + wave) % R;
      if constexpr (X) {
        const int row = (block & 3) * 8 + (lane >> 3);
        at[i] = (row * (int)o.ld + (block >> 2) * 64 + ((lane & 7) ^ swap_of(row)) * 8) * 2;
      } else {
        // the row stands in the lane's offset, k in the scalar one: what is out of range is then so by the
        // lane's offset alone
        at[i] = ((block * 16 + (lane & 15)) * (int)o.ld + (lane >> 4) * 8) * 2;
      }
    }
    if constexpr (X) {
      const int g = lane >> 4, r = (lane >> 2) & 3, q = lane & 3, swap = swap_of(g * 8 + r);
#pragma unroll
      for (int i = 0; i < 4; ++i) read[i] = g * 1024 + r * 128 + ((i * 2 + (q >> 1)) ^ swap) * 16 + (q & 1) * 8;
    }
  }

  // Copies the stage at k (the next one, for ACROSS) of every plane to LDS.
  __device__ __forceinline__ void fetch(int k, char* to, int wave) {
    if constexpr (X) {
#pragma unroll
      for (int q = 0; q < NP; ++q) rsrc[q] = window(base[q], bytes);
    }
#pragma unroll
    for (int q = 0; q < NP; ++q)
#pragma unroll
      for (int i = 0; i < N; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rsrc[q], (__attribute__((address_space(3))) void*)(to + (q * R + (i * NW + wave) % R) * 1024), 16, at[i],
            X ? 0 : k * 2, 0, 0);
    if constexpr (X) {
#pragma unroll
      for (int q = 0; q < NP; ++q) base[q] += step;
      bytes -= step * 2;
    }
  }

  // What the instruction takes of 16 rows `block` of plane q.
  __device__ __forceinline__ u32x4 fragment(const char* from, int q, int block, int lane) const {
    if constexpr (X) {
      typedef __attribute__((address_space(3))) s16x4 L;
      const char* p = from + (q * R + (block >> 2) * 4) * 1024 + read[block & 3];
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(p + 512)));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      return *reinterpret_cast<const u32x4*>(from + (q * R + block) * 1024 + lane * 16);
    }
  }
};
#endif

// acc[i][j] += blocks of D for m0 .. and n0 .., k from k_begin to k_end (multiples of 32).  lds: T::LDS
// bytes.
template <class T>
__device__ __forceinline__ void multiply(const Operand& a, const Operand& b, long batch, int m0, int n0,
                                         int k_begin, int k_end, char* lds, f32x4 (&acc)[T::TM][T::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  if (k_begin >= k_end) return;
  Side<T::BM, T::AX, T::NP, T::NW> sa(a, batch, m0, k_begin, lane, wave);
  Side<T::BN, T::BX, T::NP, T::NW> sb(b, batch, n0, k_begin, lane, wave);
  constexpr int B_AT = T::NP * T::RA * 1024;
  const auto fetch = [&](int k, char* to) {
    sa.fetch(k, to, wave);
    sb.fetch(k, to + B_AT, wave);
  };
  const auto work = [&](const char* from) {
    u32x4 fa[T::NP][T::TM], fb[T::NP][T::TN];
#pragma unroll
    for (int q = 0; q < T::NP; ++q) {
#pragma unroll
      for (int i = 0; i < T::TM; ++i) fa[q][i] = sa.fragment(from, q, wm * T::TM + i, lane);
#pragma unroll
      for (int j = 0; j < T::TN; ++j) fb[q][j] = sb.fragment(from + B_AT, q, wn * T::TN + j, lane);
    }
    __builtin_amdgcn_s_setprio(1);
    // smallest products first
#pragma unroll
    for (int s = T::NP - 1; s >= 0; --s)
#pragma unroll
      for (int q = 0; q <= s; ++q)
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
          for (int j = 0; j < T::TN; ++j) acc[i][j] = multiply_block<T::NP>(fa[q][i], fb[s - q][j], acc[i][j]);
    __builtin_amdgcn_s_setprio(0);
  };
  const int stages = (k_end - k_begin) / 32;
#pragma unroll
  for (int s = 0; s < T::RING - 1; ++s)
    if (s < stages) fetch(k_begin + s * 32, lds + s * T::STAGE);
  int slot = 0, next = T::RING - 1;
  for (int t = 0; t < stages; ++t) {
    // under way beyond this stage: min(RING - 2, stages - 1 - t) stages
    const int beyond = stages - 1 - t;
    if (beyond >= T::RING - 2) wait_copies<T::COPIES * (T::RING - 2)>();
    else if (T::RING > 3 && beyond == 1) wait_copies<T::COPIES>();
    else wait_copies<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t + T::RING - 1 < stages) fetch(k_begin + (t + T::RING - 1) * 32, lds + next * T::STAGE);
    work(lds + slot * T::STAGE);
    slot = slot + 1 == T::RING ? 0 : slot + 1;
    next = next + 1 == T::RING ? 0 : next + 1;
  }
#endif
}

}  // namespace prod
}  // namespace wino
