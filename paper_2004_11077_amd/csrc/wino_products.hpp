// Matrix products of the training operators (linear cross entropy, orthogonalised updates):
//   D[m][n] = sum_k A[m][k] B[n][k]        both operands with k contiguous
// on the bf16 matrix pipe (v_mfma_f32_16x16x32_bf16, fp32 accumulation).
//
// An operand is NP planes of bf16 that add up to its values.  NP = 1: bf16 values as they stand.
// NP = 3: an fp32 value x as h + m + l, h its upper 8 significant bits (cut, so that nothing
// overflows), m the rest rounded to bf16, l what is then left, which is a bf16 value: h + m + l = x
// exactly.  Of the nine products of two such sums the six largest are taken; the three left out are
// below 2^-22 of the term with the signs of m and l, which are as often positive as negative.
// NP = 2: fp16 instead of bf16, x as fp16(x) + fp16(x - fp16(x)), 22 significant bits; three of four
// products.  Its narrow exponent wants x times a power of two known beforehand, so that the largest
// magnitude is 2^15 or below; what is smaller than 2^-18 of that keeps 2^-40 of it.
// Products of two such values are exact in fp32, so a sum is as good as one of fp32 products, at six
// (three) matrix instructions of 2.5 PFLOP/s instead of one fp32 instruction of 0.157 PFLOP/s.
//
// Tile: BM x BN of D per work group, WM x WN waves, 16 x 16 blocks of D per instruction.  A stage of
// 32 k of every plane is copied from memory straight into LDS (buffer_load ... lds), in the order in
// which the instruction takes its operand: 16 rows x 32 k are one KiB, lane l's 16 bytes at 16 l.
// Reads are then conflict-free and need no address arithmetic, and an operand that lies in plain
// rows needs no rearrangement, because a lane may fetch from anywhere.  Planes that are written for
// a product alone lie in that order in memory too (BLOCKED), whole lines a copy.  RING buffers, RING - 1
// stages under way: a wave waits until its own copies of a stage have landed (counted, so that the
// later stages' stay under way), the barrier then says so of all waves, and also that the buffer of
// the stage before may be filled again.  Rows past the last one lie outside the buffer descriptor
// and read as zeros; K is a multiple of 32, the caller pads with zeros.  A work group's first row
// exists, and kMaxLd bounds the offsets within a tile to 31 bits.
// 65536 x 4096 x 2048, bf16 (the best plain library product there: 1180 TFLOP/s):
//   128 x 128 tiles, 4 waves, two buffers of 64 k, all copies waited for   582 TFLOP/s
//   256 x 256, 8 waves, the same                                            877
//   256 x 256, 8 waves, ring of four, counted waits                         987
//   and the multiplying wave before the fetching one (s_setprio)           1052
// 256 x 256 and 8 waves read 12 KiB of LDS a wave for 32 instructions of 16 cycles, 1536 of a
// stage's 2048 cycles of LDS at both stages' worth; smaller tiles are bound by it.
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

constexpr long kMaxLd = 1L << 21;   // elements between rows: 256 rows of it are 2^30 bytes

// Rows of one operand: plane q, batch b, row r, element k at p + q plane + b batch + r ld + k; BLOCKED:
// 16 rows x 32 k a KiB, lane l of 64 holding row l % 16 and k of l / 16 (8 of them), blocks of one row of
// blocks ld elements long, `rows` rounded up to whole blocks.
struct Operand {
  const uint16_t* p;
  long ld, plane, batch;
  int rows;
};
// Element of blocked planes whose rows have kb blocks.
__host__ __device__ __forceinline__ long blocked(int row, int k, int kb) {
  return ((long)(row >> 4) * kb + (k >> 5)) * 512 + ((k & 31) >> 3) * 128 + (row & 15) * 8 + (k & 7);
}

__device__ __forceinline__ uint16_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ float bf16_value(uint16_t b) {
  return __builtin_bit_cast(float, (uint32_t)b << 16);
}

__device__ __forceinline__ uint16_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
__device__ __forceinline__ float f16_value(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }

// x as NP 16-bit values (see above).
template <int NP>
__device__ __forceinline__ void cut(float x, uint16_t (&out)[NP]) {
  if constexpr (NP == 1) {
    out[0] = bf16_bits(x);
  } else if constexpr (NP == 2) {
    out[0] = f16_bits(x);
    out[1] = f16_bits(x - f16_value(out[0]));
  } else {
    out[0] = (uint16_t)(__builtin_bit_cast(uint32_t, x) >> 16);
    const float r = x - bf16_value(out[0]);
    out[1] = bf16_bits(r);
    out[2] = bf16_bits(r - bf16_value(out[1]));
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

template <int BM_, int BN_, int WM_, int WN_, int NP_, int RING_, bool BLOCKED_ = false>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NP = NP_, RING = RING_;
  static constexpr bool BLOCKED = BLOCKED_;
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 blocks per wave
  static constexpr int RA = BM / 16, RB = BN / 16;             // 16-row blocks of the operands
  static constexpr int STAGE = NP * (RA + RB) * 1024;          // bytes
  static constexpr int LDS = RING * STAGE;
  // copies of a stage per wave and plane; where there are fewer blocks than waves, several waves
  // copy the same one, so that all count alike
  static constexpr int NA = (RA + NW - 1) / NW, NB = (RB + NW - 1) / NW;
  static constexpr int COPIES = NP * (NA + NB);
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && RING >= 2 && LDS <= 160 * 1024);
  static_assert((RA % NW == 0 || NW % RA == 0) && (RB % NW == 0 || NW % RB == 0));
  static_assert(COPIES * (RING - 2) < 64);   // what a counted wait can say
};

#if defined(__HIP_DEVICE_COMPILE__)
// Buffer descriptor of up to `tile_rows` rows from row r0 of one plane; `k` elements of the last row.
template <bool BLOCKED>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const Operand& o, int plane, long batch, int r0,
                                                          int tile_rows, int k) {
  constexpr int PER = BLOCKED ? 16 : 1;   // rows that ld spans
  const uint16_t* p = o.p + plane * o.plane + batch * o.batch + (long)(r0 / PER) * o.ld;
  int rows = o.rows - r0;
  rows = rows < tile_rows ? rows : tile_rows;
  const long bytes = rows <= 0 ? 0 : BLOCKED ? (long)((rows + 15) / 16) * o.ld * 2 : ((long)(rows - 1) * o.ld + k) * 2;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, (int)bytes, 0x00020000);
}

// Waits until at most N of this wave's copies are under way.  Its LDS reads have all been used by then;
// saying so costs nothing and makes the barrier behind it mean that the buffer is free.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
#endif

// acc[i][j] += blocks of D for rows m0 .. of A and n0 .. of B, k from k_begin to k_end (multiples of
// 32).  lds: T::LDS bytes.
template <class T>
__device__ __forceinline__ void multiply(const Operand& a, const Operand& b, long batch, int m0, int n0,
                                         int k_begin, int k_end, int k_total, char* lds,
                                         f32x4 (&acc)[T::TM][T::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  __amdgpu_buffer_rsrc_t ra[T::NP], rb[T::NP];
#pragma unroll
  for (int q = 0; q < T::NP; ++q) {
    ra[q] = rows_of<T::BLOCKED>(a, q, batch, m0, T::BM, k_total);
    rb[q] = rows_of<T::BLOCKED>(b, q, batch, n0, T::BN, k_total);
  }
  // LDS of a stage: [operand][plane][16 rows][1 KiB].  The row stands in the lane's offset, k in the
  // scalar one: what is out of range is then so by the lane's offset alone.
  int at_a[T::NA], at_b[T::NB];
#pragma unroll
  for (int i = 0; i < T::NA; ++i)
    at_a[i] = T::BLOCKED ? ((i * T::NW + wave) % T::RA * (int)a.ld + lane * 8) * 2
                         : (((i * T::NW + wave) % T::RA * 16 + (lane & 15)) * (int)a.ld + (lane >> 4) * 8) * 2;
#pragma unroll
  for (int i = 0; i < T::NB; ++i)
    at_b[i] = T::BLOCKED ? ((i * T::NW + wave) % T::RB * (int)b.ld + lane * 8) * 2
                         : (((i * T::NW + wave) % T::RB * 16 + (lane & 15)) * (int)b.ld + (lane >> 4) * 8) * 2;
  constexpr int kStep = T::BLOCKED ? 32 : 2;   // bytes from one k to the next, 32 of them at a time
  const auto fetch = [&](int k, char* to) {
#pragma unroll
    for (int q = 0; q < T::NP; ++q) {
#pragma unroll
      for (int i = 0; i < T::NA; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            ra[q], (__attribute__((address_space(3))) void*)(to + (q * T::RA + (i * T::NW + wave) % T::RA) * 1024),
            16, at_a[i], k * kStep, 0, 0);
#pragma unroll
      for (int i = 0; i < T::NB; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rb[q],
            (__attribute__((address_space(3))) void*)(to + (T::NP * T::RA + q * T::RB + (i * T::NW + wave) % T::RB) * 1024),
            16, at_b[i], k * kStep, 0, 0);
    }
  };
  const auto work = [&](const char* from) {
    u32x4 fa[T::NP][T::TM], fb[T::NP][T::TN];
#pragma unroll
    for (int q = 0; q < T::NP; ++q) {
#pragma unroll
      for (int i = 0; i < T::TM; ++i)
        fa[q][i] = *reinterpret_cast<const u32x4*>(from + (q * T::RA + wm * T::TM + i) * 1024 + lane * 16);
#pragma unroll
      for (int j = 0; j < T::TN; ++j)
        fb[q][j] = *reinterpret_cast<const u32x4*>(from + (T::NP * T::RA + q * T::RB + wn * T::TN + j) * 1024 + lane * 16);
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
          for (int j = 0; j < T::TN; ++j)
            acc[i][j] = multiply_block<T::NP>(fa[q][i], fb[s - q][j], acc[i][j]);
    __builtin_amdgcn_s_setprio(0);
  };
  if (k_begin >= k_end) return;
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
