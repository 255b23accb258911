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
// PFLOP/s instead of one fp32 instruction of 0.157 PFLOP/s.  NP = 3: fp32 values as they stand, cut into
// three bf16 values of 8 bits each when they are read from LDS, and six of nine products: twice the
// instructions and the cutting for every tile (as many cycles again: 59 x 4081 x 25462 takes 179 us where its
// 416 MB would pass in 86), but no planes to be written and read and no power of two
// to be known.  It is for operands that are read about once.
//
// Two planes lie together, 32 elements of the one and then 32 of the other: 128 bytes, a cache line.
//
// Tile: BM x BN of D per work group, WM x WN waves, 16 x 16 blocks of D per instruction, for which a
// lane holds eight consecutive k of one row of an operand.  A stage, 64 k of one plane or 32 of two, is
// copied from memory straight into LDS (buffer_load ... lds), eight rows of 128 bytes a wave's copy: whole
// lines (with 16 rows of 64 bytes a copy, lines that are fetched twice: 0.7 of the rate).  A lane's 16
// bytes land behind the lane before's, but a lane may fetch from anywhere, so the 16-byte pieces of a row
// change places in such a way that what a read touches lies in different banks:
//   * k along the rows of the operand in memory: lane l of the instruction reads piece l / 16 (+ 4 for the
//     second 32 k or plane) of row l % 16; piece c of row r lies at c ^ (r % 8).
//   * k across the rows (AX, BX): the rows of the copy are k.  ds_read_b64_tr_b16 hands a lane four
//     consecutive k of its m; piece c of row k lies at c ^ swap_of(k).
// No operand is therefore ever transposed in memory.  RING buffers, RING - 1 stages under way: a wave
// waits until its own copies of a stage have landed (counted, so that the later stages' stay under
// way), the barrier then says so of all waves, and also that the buffer of the stage before may be
// filled again.  What lies outside an operand lies outside its buffer descriptor and reads as zeros; k
// runs in whole stages: along rows the caller pads with zeros, but for fp32 values as they stand, whose
// last stage may be a part of one (wino_product_sources.hpp).  A work group's first row exists, and
// kMaxLd bounds the offsets within a stage to 31 bits.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "wino_kernels.hpp"
#include "wino_product_sources.hpp"
#include "wino_train_rules.hpp"

namespace wino {
namespace prod {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// One operand: `rows` rows of `cols` elements, batch b, row r at p + b batch + r ld, element e of plane q
// there at place<NP>(e) + 32 q; fp32 (NP = 3): at 2 e, strides in 16-bit units too.  k along the rows: m or n is r, k is e.  Across: k is r, m or n is e.
struct Operand {
  const uint16_t* p;
  long ld, batch;
  int rows, cols;
};
template <int NP>
__host__ __device__ __forceinline__ int place(int e) {
  return NP == 1 ? e : (e >> 5) * 64 + (e & 31);
}

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

// Two fp32 values as bf16 values, the first in the lower half.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// Eight fp32 values as three times eight bf16 values: the upper 8 bits cut off, so that nothing overflows,
// the rest rounded, and what is then left, which is a bf16 value: together x exactly.  By pairs: 5.5
// instructions a value, which are as many of the kernel's cycles as the matrix instructions are.
__device__ __forceinline__ void cut_three(const f32x4 (&x)[2], u32x4 (&out)[3]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[i >> 1][(i & 1) * 2], b = x[i >> 1][(i & 1) * 2 + 1];
    const uint32_t ha = __builtin_bit_cast(uint32_t, a) & 0xffff0000u, hb = __builtin_bit_cast(uint32_t, b) & 0xffff0000u;
    const float ra = a - __builtin_bit_cast(float, ha), rb = b - __builtin_bit_cast(float, hb);
    const uint32_t mid = bf16_pair(ra, rb);
    out[0][i] = ha >> 16 | hb;
    out[1][i] = mid;
    out[2][i] = bf16_pair(ra - __builtin_bit_cast(float, mid << 16), rb - __builtin_bit_cast(float, mid & 0xffff0000u));
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

// Work group of a grid of `all` -> its place.  Consecutive work groups go round robin over the 8 XCDs;
// each XCD gets a run of places, so that neighbours share its L2.
__device__ __forceinline__ int place_of_group(int b, int all) {
  const int per = all / 8;
  return b < per * 8 ? (b & 7) * per + (b >> 3) : b;
}
// Place -> tile (m, n): bands of eight tiles m, whose rows stay in the L2 while those of n pass.
__device__ __forceinline__ void tile_at(int b, int tiles_m, int tiles_n, int& m, int& n) {
  const int band = b / (8 * tiles_n), rest = b - band * 8 * tiles_n;
  const int wide = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
  m = band * 8 + rest % wide;
  n = rest / wide;
}

template <int BM_, int BN_, int WM_, int WN_, int NP_, int RING_, bool AX_ = false, bool BX_ = false>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NP = NP_, RING = RING_;
  static constexpr bool AX = AX_, BX = BX_;                    // k across the rows of A, of B
  static constexpr int NW = WM * WN, THREADS = 64 * NW;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 blocks per wave
  static constexpr int K = NP == 1 ? 64 : 32;                  // k of a stage
  static constexpr int RA = BM / 8, RB = BN / 8;               // KiB of a stage of the operands
  static constexpr int STAGE = (RA + RB) * 1024;               // bytes
  static constexpr int LDS = RING * STAGE;
  static constexpr int COPIES = (RA + RB) / NW;                // of a stage per wave
  static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && RING >= 2 && LDS <= 160 * 1024);
  static_assert(RA % NW == 0 && RB % NW == 0 && BM % 64 == 0 && BN % 64 == 0);
  static_assert(COPIES * (RING - 2) < 64);   // what a counted wait can say
};

// Products of few tiles and k along the rows of both operands, where waiting counts: 32 x 32 of D a
// work group.  Its WAVES waves take every WAVES-th line of k, fragments straight from memory into
// registers, many lines under way and no barrier in the loop; their sums are joined in LDS, after which
// each of the first four waves has one of the four 16 x 16 blocks, as if the tile were 2 x 2 waves.
template <int NP_, int WAVES_ = 4>
struct Few {
  static constexpr int BM = 32, BN = 32, WM = 2, WN = 2, NP = NP_, WAVES = WAVES_, TM = 1, TN = 1;
  static constexpr int THREADS = 64 * WAVES, K = NP == 1 ? 64 : 32, LDS = WAVES * 4096;
};
template <class T>
constexpr bool is_few = false;
template <int NP, int WAVES>
constexpr bool is_few<Few<NP, WAVES>> = true;

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

// Places of the 16-byte pieces of a row k that the operand's k runs across.  A read touches rows 8 g + r
// (+ 4) of four lane groups g, four r each, two neighbouring pieces of a row; rows are 128 bytes, so the
// half of the banks goes by r % 2, and within it the four places by r / 2 and g % 2.
__device__ __forceinline__ int swap_of(int k) { return ((k >> 1) & 1) * 2 + ((k >> 3) & 1) * 4; }

// One operand's side of a tile: SIDE rows (m or n), X: k across.
template <int SIDE, bool X, int NP, int NW>
struct Side {
  static constexpr int K = NP == 1 ? 64 : 32, KG = K / 8, N = SIDE / 8 / NW;
  static constexpr int UNITS = NP == 1 ? 1 : 2;   // 16-bit units of an element
  static constexpr int PARTS = NP == 3 ? 3 : 2;   // what a fragment comes in
  const uint16_t* base;
  long bytes, step;          // from the base to the operand's end; across: elements of a stage
  __amdgpu_buffer_rsrc_t rsrc;
  int at[N];                 // a copy's source, in bytes from the base
  int read[X ? 4 : 2];       // a lane's places in a stage
  int cols, value;           // value: fp32 along rows, the stage's k that the lane copies from

  // own: the wave's first block of 16 rows.
  __device__ __forceinline__ Side(const Operand& o, long batch, int first, int k, int own, int lane, int wave) {
    const long start = X ? (long)k * o.ld + first * UNITS : (long)first * o.ld;
    base = o.p + batch * o.batch + start;
    if constexpr (X) {
      bytes = ((long)(o.rows - 1) * o.ld + (long)o.cols * UNITS - start) * 2;
      step = K * o.ld;
    } else {
      int rows = o.rows - first;
      rows = rows < SIDE ? rows : SIDE;
      bytes = ((long)(rows - 1) * o.ld + (long)o.cols * UNITS) * 2;
      step = 0;
      rsrc = window(base, bytes);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int block = i * NW + wave;
      if constexpr (X) {
        const int row = block % KG * 8 + (lane >> 3);
        at[i] = (row * (int)o.ld + block / KG * 64 + ((lane & 7) ^ swap_of(row)) * 8) * 2;
      } else {
        // the row stands in the lane's offset, k in the scalar one: what is out of range is then so by the
        // lane's offset alone
        at[i] = ((block * 8 + (lane >> 3)) * (int)o.ld + ((lane & 7) ^ (lane >> 3)) * 8) * 2;
      }
    }
    cols = o.cols;
    value = copied_value(lane);
    if constexpr (X && NP == 3) {
      // place i: half i / 2 of 32 values, rows with bit 1 of k as i % 2
      const int g = lane >> 4, e = lane & 15;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        read[i] = g * 1024 + (((i >> 1) * 4 + (e >> 2)) ^ ((i & 1) * 2 + (g & 1) * 4)) * 16 + (e & 3) * 4;
    } else if constexpr (X) {
      const int g = lane >> 4, r = (lane >> 2) & 3, q = lane & 3, swap = swap_of(g * 8 + r);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int place = NP == 1 ? (own + i) & 3 : i;   // one plane: of the wave's block i
        read[i] = g * 1024 + r * 128 + ((place * 2 + (q >> 1)) ^ swap) * 16 + (q & 1) * 8;
      }
    } else {
      const int r = lane & 7;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        read[i] = (lane & 15) * 128 + ((NP == 3 ? (lane >> 4) * 2 + i : i * 4 + (lane >> 4)) ^ r) * 16;
    }
  }

  // Copies the stage at k (the next one, for k across) to LDS.
  __device__ __forceinline__ void fetch(int k, char* to, int wave) {
    if constexpr (X) rsrc = window(base, bytes);
    const auto copy = [&](int i, int lane_at, int scalar_at) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(to + (i * NW + wave) * 1024), 16, lane_at, scalar_at, 0, 0);
    };
    if (NP == 3 && !X && k + K > cols) {
#pragma unroll
      for (int i = 0; i < N; ++i) copy(i, source_at(at[i], value, k, cols).lane, 0);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) copy(i, at[i], X ? 0 : k * 2 * UNITS);
    }
    if constexpr (X) {
      base += step;
      bytes -= step * 2;
    }
  }

  // What the instruction takes of 16 rows, block own + i, of the stage at k: the two parts of 32 k of one plane, the two
  // planes, or the three pieces of fp32 values.
  __device__ __forceinline__ void fragment(const char* from, int own, int i, int k, int lane, u32x4 (&out)[PARTS]) const {
    const int block = own + i;
    if constexpr (NP == 3) {
      f32x4 x[2];
      if constexpr (X) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          x[j >> 2][j & 3] = *reinterpret_cast<const float*>(from + (block >> 1) * 4096 + j * 128 + read[(block & 1) * 2 + ((j >> 1) & 1)]);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = *reinterpret_cast<const f32x4*>(from + block * 2048 + read[h]);
        if (k + 32 > cols)   // the next row's values, or nothing's
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (k + (lane >> 4) * 8 + e >= cols) x[e >> 2][e & 3] = 0;
      }
      cut_three(x, out);
    } else {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        if constexpr (X) {
          typedef __attribute__((address_space(3))) s16x4 L;
          const char* p = NP == 1 ? from + ((block >> 2) * 8 + sub * 4) * 1024 + read[i & 3]
                                  : from + (block >> 1) * 4096 + read[sub * 2 + (block & 1)];
          const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p));
          const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(p + 512)));
          out[sub] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
          out[sub] = *reinterpret_cast<const u32x4*>(from + block * 2048 + read[sub]);
        }
      }
    }
  }
};
#endif

// Two planes: upper and lower, lower and upper, upper and upper; one: its two parts of 32 k each; three
// pieces: the six largest products, the smallest first.
template <int NP, int TM, int TN, int PARTS>
__device__ __forceinline__ void multiply_parts(const u32x4 (&a)[TM][PARTS], const u32x4 (&b)[TN][PARTS], f32x4 (&acc)[TM][TN]) {
#pragma unroll
  for (int s = 0; s < NP * (NP + 1) / 2 + (NP == 1); ++s) {
    constexpr int P3[] = {0, 1, 2, 0, 1, 0}, Q3[] = {2, 1, 0, 1, 0, 0};
    const int p = NP == 1 ? s : NP == 2 ? s == 1 : P3[s], q = NP == 1 ? s : NP == 2 ? s == 0 : Q3[s];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = multiply_block<NP>(a[i][p], b[j][q], acc[i][j]);
  }
}

#if defined(__HIP_DEVICE_COMPILE__)
template <class T>
__device__ __forceinline__ void multiply_few(const Operand& a, const Operand& b, long batch, int m0, int n0,
                                             int k_begin, int k_end, char* lds, f32x4& out) {
  constexpr int DEPTH = 4, UNITS = T::NP == 1 ? 1 : 2, PARTS = T::NP == 3 ? 3 : 2;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int left_a = a.rows - m0 < 32 ? a.rows - m0 : 32, left_b = b.rows - n0 < 32 ? b.rows - n0 : 32;
  const auto ra = window(a.p + batch * a.batch + (long)m0 * a.ld, ((left_a - 1) * a.ld + (long)a.cols * UNITS) * 2);
  const auto rb = window(b.p + batch * b.batch + (long)n0 * b.ld, ((left_b - 1) * b.ld + (long)b.cols * UNITS) * 2);
  // a lane's two 16-byte pieces of a line: fp32's eight values, or eight of each part
  constexpr int STEP = T::NP == 3 ? 16 : 8, HALF = T::NP == 3 ? 16 : 64;
  const int at_a = ((lane & 15) * (int)a.ld + (lane >> 4) * STEP) * 2, at_b = ((lane & 15) * (int)b.ld + (lane >> 4) * STEP) * 2;
  const int next_a = 32 * (int)a.ld, next_b = 32 * (int)b.ld;   // 16 rows on, bytes
  f32x4 acc[2][2] = {};
  const int lines = k_end / T::K;
  for (int l = k_begin / T::K + wave; l < lines; l += DEPTH * T::WAVES) {
    u32x4 fa[DEPTH][2][2], fb[DEPTH][2][2];   // [line][16 rows][piece]
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      // lines beyond the last one: out of the window, zeros
      const int line = l + d * T::WAVES;
      const auto load = [&](auto rsrc, int at, int cols, int q) {
        Source s{kRefused, 0};
        if (line < lines) s = T::NP == 3 ? source_at(at, loaded_value(lane, q), line * 32, cols) : Source{at, line * 128};
        return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, s.lane, s.scalar, 0));
      };
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fa[d][i][q] = load(ra, at_a + i * next_a + q * HALF, a.cols, q);
          fb[d][i][q] = load(rb, at_b + i * next_b + q * HALF, b.cols, q);
        }
    }
    __builtin_amdgcn_sched_barrier(0);   // all loads before the first product
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      if constexpr (T::NP == 3) {
        u32x4 pa[2][PARTS], pb[2][PARTS];
        const auto pieces = [&](const u32x4 (&from)[2], int cols, u32x4 (&out)[PARTS]) {
          f32x4 x[2] = {__builtin_bit_cast(f32x4, from[0]), __builtin_bit_cast(f32x4, from[1])};
          const int k = (l + d * T::WAVES) * 32;
          if (k + 32 > cols)   // the next row's values, or nothing's
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (k + (lane >> 4) * 8 + e >= cols) x[e >> 2][e & 3] = 0;
          cut_three(x, out);
        };
#pragma unroll
        for (int i = 0; i < 2; ++i) pieces(fa[d][i], a.cols, pa[i]), pieces(fb[d][i], b.cols, pb[i]);
        multiply_parts<3>(pa, pb, acc);
      } else {
        multiply_parts<T::NP>(fa[d], fb[d], acc);
      }
    }
  }
  f32x4* join = reinterpret_cast<f32x4*>(lds);   // [wave][block][lane]
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) join[(wave * 4 + j * 2 + i) * 64 + lane] = acc[i][j];
  __syncthreads();
  if (wave < 4) {   // block (wave % 2, wave / 2)
    out = join[wave * 64 + lane];
#pragma unroll
    for (int w = 1; w < T::WAVES; ++w) out += join[(w * 4 + wave) * 64 + lane];
  }
}
#endif

// acc[i][j] += blocks of D for m0 .. and n0 .., k from k_begin to k_end (multiples of T::K).  lds: T::LDS
// bytes.
template <class T>
__device__ __forceinline__ void multiply(const Operand& a, const Operand& b, long batch, int m0, int n0,
                                         int k_begin, int k_end, char* lds, f32x4 (&acc)[T::TM][T::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (is_few<T>) {
    multiply_few<T>(a, b, batch, m0, n0, k_begin, k_end, lds, acc[0][0]);
  } else {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  if (k_begin >= k_end) return;
  Side<T::BM, T::AX, T::NP, T::NW> sa(a, batch, m0, k_begin, wm * T::TM, lane, wave);
  Side<T::BN, T::BX, T::NP, T::NW> sb(b, batch, n0, k_begin, wn * T::TN, lane, wave);
  constexpr int B_AT = T::RA * 1024;
  const auto fetch = [&](int k, char* to) {
    sa.fetch(k, to, wave);
    sb.fetch(k, to + B_AT, wave);
  };
  const auto some = [&](const char* from, int k, auto& fa, auto& part) {
    u32x4 fb[T::TN][decltype(sb)::PARTS];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(fa) / sizeof(fa[0])); ++i) sa.fragment(from, wm * T::TM, i, k, lane, fa[i]);
#pragma unroll
    for (int j = 0; j < T::TN; ++j) sb.fragment(from + B_AT, wn * T::TN, j, k, lane, fb[j]);
    __builtin_amdgcn_s_setprio(1);
    multiply_parts<T::NP>(fa, fb, part);
    __builtin_amdgcn_s_setprio(0);
  };
  // Cutting fp32 values costs as much as multiplying them: not done for blocks of 16 rows m that do not exist.
  const int blocks = T::NP == 3 ? ((T::AX ? a.cols : a.rows) - m0 + 15) / 16 - wm * T::TM : T::TM;
  const auto work = [&](const char* from, int k) {
    if (T::NP < 3 || blocks > 1) {
      u32x4 fa[T::TM][decltype(sa)::PARTS];
      some(from, k, fa, acc);
    } else if (blocks == 1) {
      u32x4 fa[1][decltype(sa)::PARTS];
      some(from, k, fa, reinterpret_cast<f32x4(&)[1][T::TN]>(acc));
    }
  };
  const int stages = (k_end - k_begin) / T::K;
#pragma unroll
  for (int s = 0; s < T::RING - 1; ++s)
    if (s < stages) fetch(k_begin + s * T::K, lds + s * T::STAGE);
  int slot = 0, next = T::RING - 1;
  for (int t = 0; t < stages; ++t) {
    // under way beyond this stage: min(RING - 2, stages - 1 - t) stages
    const int beyond = stages - 1 - t;
    if (beyond >= T::RING - 2) wait_copies<T::COPIES * (T::RING - 2)>();
    else if (T::RING > 3 && beyond == 1) wait_copies<T::COPIES>();
    else wait_copies<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t + T::RING - 1 < stages) fetch(k_begin + (t + T::RING - 1) * T::K, lds + next * T::STAGE);
    work(lds + slot * T::STAGE, k_begin + t * T::K);
    slot = slot + 1 == T::RING ? 0 : slot + 1;
    next = next + 1 == T::RING ? 0 : next + 1;
  }
  }
#endif
}

}  // namespace prod
}  // namespace wino
