// Matrix products of the training operators (linear cross entropy, orthogonalised updates):
//   D[m][n] = sum_k A[m][k] B[n][k]        both operands with k contiguous
// on the bf16 matrix pipe (v_mfma_f32_16x16x32_bf16, fp32 accumulation).
//
// An operand is NP planes of bf16 that add up to its values.  NP = 1: bf16 values as they stand.
// NP = 3: an fp32 value x as h + m + l, h its upper 8 significant bits (cut, so that nothing
// overflows), m the rest rounded to bf16, l what is then left, which is a bf16 value: h + m + l = x
// exactly.  Of the nine products of two such sums the six largest are taken; the three left out are
// below 2^-22 of the term with the signs of m and l, which are as often positive as negative.
// NP = 2: x as bf16(x) + bf16(x - bf16(x)), 16 significant bits; three of four products.
// Products of two bf16 values are exact in fp32, so a sum is as good as one of fp32 products, at six
// matrix instructions of 2.5 PFLOP/s instead of one fp32 instruction of 0.157 PFLOP/s.
//
// Tile: BM x BN of D per work group, WM x WN waves, 16 x 16 blocks of D per instruction.  A stage of
// BK of every plane is copied from memory straight into LDS (buffer_load ... lds), in the order in
// which the instruction takes its operand: 16 rows x 32 k are one KiB, lane l's 16 bytes at 16 l.
// Reads are then conflict-free and need no address arithmetic, and the layout in memory stays
// plain rows, because a lane may fetch from anywhere.  Two buffers: the next stage is under way
// while this one is multiplied.  Rows past the last one lie outside the buffer descriptor and
// read as zeros; K is a multiple of BK, the caller pads with zeros.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "wino_kernels.hpp"

namespace wino {
namespace prod {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr long kMaxLd = 1L << 21;   // elements between rows: 256 rows of it are 2^30 bytes

// Rows of one operand: plane q, batch b, row r, element k at p + q plane + b batch + r ld + k.
struct Operand {
  const uint16_t* p;
  long ld, plane, batch;
  int rows;
};

__device__ __forceinline__ uint16_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ float bf16_value(uint16_t b) {
  return __builtin_bit_cast(float, (uint32_t)b << 16);
}

// x as NP bf16 values (see above).
template <int NP>
__device__ __forceinline__ void cut(float x, uint16_t (&out)[NP]) {
  if constexpr (NP == 1) {
    out[0] = bf16_bits(x);
  } else if constexpr (NP == 2) {
    out[0] = bf16_bits(x);
    out[1] = bf16_bits(x - bf16_value(out[0]));
  } else {
    out[0] = (uint16_t)(__builtin_bit_cast(uint32_t, x) >> 16);
    const float r = x - bf16_value(out[0]);
    out[1] = bf16_bits(r);
    out[2] = bf16_bits(r - bf16_value(out[1]));
  }
}

template <int BM_, int BN_, int WM_, int WN_, int NP_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NP = NP_;
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int BK = NP == 1 ? 64 : 32;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 blocks per wave
  static constexpr int STAGE = NP * (BM + BN) * BK * 2;        // bytes
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0);
};

#if defined(__HIP_DEVICE_COMPILE__)
// Buffer descriptor of up to `tile_rows` rows from row r0 of one plane; `k` elements of the last row.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const Operand& o, int plane, long batch, int r0,
                                                          int tile_rows, int k) {
  const uint16_t* p = o.p + plane * o.plane + batch * o.batch + (long)r0 * o.ld;
  int rows = o.rows - r0;
  rows = rows < tile_rows ? rows : tile_rows;
  const long bytes = rows > 0 ? ((long)(rows - 1) * o.ld + k) * 2 : 0;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, (int)bytes, 0x00020000);
}
#endif

// acc[i][j] += blocks of D for rows m0 .. of A and n0 .. of B, k from k_begin to k_end (multiples of
// BK).  lds: 2 STAGE bytes.
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
    ra[q] = rows_of(a, q, batch, m0, T::BM, k_total);
    rb[q] = rows_of(b, q, batch, n0, T::BN, k_total);
  }
  // LDS of a stage: [operand][plane][k / 32][16 rows][1 KiB].  The row stands in the lane's offset, k
  // in the scalar one: what is out of range is then so by the lane's offset alone.
  constexpr int KB = T::BK / 32, RA = T::BM / 16, RB = T::BN / 16;
  constexpr int NA = (RA + T::NW - 1) / T::NW, NB = (RB + T::NW - 1) / T::NW;
  int at_a[NA], at_b[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i)
    at_a[i] = (((i * T::NW + wave) * 16 + (lane & 15)) * (int)a.ld + (lane >> 4) * 8) * 2;
#pragma unroll
  for (int i = 0; i < NB; ++i)
    at_b[i] = (((i * T::NW + wave) * 16 + (lane & 15)) * (int)b.ld + (lane >> 4) * 8) * 2;
  const auto fetch = [&](int k, char* to) {
#pragma unroll
    for (int q = 0; q < T::NP; ++q)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int i = 0; i < NA; ++i) {
          const int r = i * T::NW + wave;
          if (RA % T::NW == 0 || r < RA)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                ra[q], (__attribute__((address_space(3))) void*)(to + ((q * KB + kb) * RA + r) * 1024), 16,
                at_a[i], (k + kb * 32) * 2, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int r = i * T::NW + wave;
          if (RB % T::NW == 0 || r < RB)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rb[q], (__attribute__((address_space(3))) void*)(to + T::NP * KB * RA * 1024 + ((q * KB + kb) * RB + r) * 1024), 16,
                at_b[i], (k + kb * 32) * 2, 0, 0);
        }
      }
  };
  const auto work = [&](const char* from) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      bf16x8 fa[T::NP][T::TM], fb[T::NP][T::TN];
#pragma unroll
      for (int q = 0; q < T::NP; ++q) {
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
          fa[q][i] = *reinterpret_cast<const bf16x8*>(from + ((q * KB + kb) * RA + wm * T::TM + i) * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
          fb[q][j] = *reinterpret_cast<const bf16x8*>(from + T::NP * KB * RA * 1024 +
                                                      ((q * KB + kb) * RB + wn * T::TN + j) * 1024 + lane * 16);
      }
      // smallest products first
#pragma unroll
      for (int s = T::NP - 1; s >= 0; --s)
#pragma unroll
        for (int q = 0; q <= s; ++q)
#pragma unroll
          for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[q][i], fb[s - q][j], acc[i][j], 0, 0, 0);
    }
  };
  if (k_begin >= k_end) return;
  fetch(k_begin, lds);
  int buffer = 0;
  for (int k = k_begin; k < k_end; k += T::BK) {
    __syncthreads();   // waits for this stage's copies; every wave is done with the other buffer
    if (k + T::BK < k_end) fetch(k + T::BK, lds + (buffer ^ 1) * T::STAGE);
    work(lds + buffer * T::STAGE);
    buffer ^= 1;
  }
#endif
}

}  // namespace prod
}  // namespace wino
