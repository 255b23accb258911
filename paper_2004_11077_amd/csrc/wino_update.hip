// Orthogonalising a weight gradient by Newton-Schulz products:
//
//   X = G / (|G|_F + eps);  `steps` times  A = X X^T,  X <- a X + (b A + c A A) X;  O = scale X
//
// on the smaller side's products (a taller matrix is taken across).  Three products a step
// (wino_products.hpp): A = X X^T, the polynomial P = a I + b A + c A A from A, which is symmetric, and
// the new X = P X.  Every product leaves its result cut into the two fp16 planes that the next one
// takes.  A step multiplies small singular values by a and the errors of earlier steps with them, by
// 3.4^4 in all for the usual coefficients, so bf16 results need the second plane as well.
//
// What bounds it: the matrix pipe for large matrices, launches for small ones, of which there are three or
// four a step.  6144 x 1536: 1.09 ms where the 236 GFLOP of fp32 products need 0.54 at the rate of the
// library's large bf16 product over three; 3 x 512 x 4608, bf16: 368 us for 0.13 ms of products; 3 x 256 x
// 2304: 153 us; 4 x 64 x 576: 92 us for 17 launches.
//
// Powers of two that bring X, A and P into fp16's range are known on the host: no singular value of X
// exceeds one at first, nor, after a step, the largest |a s + b s^3 + c s^5| of those before it, and no
// entry exceeds the largest singular value.  (2^15 is half of what fp16 holds.)
#include <cmath>

#include "wino_products.hpp"
#include "wino_train.hpp"

namespace wino {
namespace {

using namespace prod;
using namespace update;

__device__ __forceinline__ float value(const void* p, long i, int bf16) {
  return bf16 ? bf16_value(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// Sums of squares of a matrix in 64 bits: no square over- or underflows.
__global__ __launch_bounds__(256) void k_update_norm(const void* __restrict__ g, UpdateArgs a,
                                                      double* __restrict__ norms) {
  __shared__ double lds[4];
  const long base = blockIdx.y * a.g_batch;
  double s = 0;
  const auto take = [&](long at) {
    const double v = value(g, base + at, a.g_bf16);
    s += v * v;
  };
  if (a.g_stride == a.cols) {   // one run of values
    const long items = (long)a.rows * a.cols;
#pragma unroll 8
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < items; i += kNormParts * 256) take(i);
  } else {
    for (int r = blockIdx.x; r < a.rows; r += kNormParts)
      for (int c = threadIdx.x; c < a.cols; c += 256) take(r * a.g_stride + c);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) norms[blockIdx.y * kNormParts + blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}

// fp16 planes of a matrix, rows of ld elements (whole lines, zeros behind the matrix); 2^e times the
// values.
struct Planes {
  uint16_t* p;
  long batch;
  int ld, e;
  __device__ __forceinline__ uint16_t* at(int z, int row, int k) const {
    return p + z * batch + (long)row * ld * 2 + place<2>(k);
  }
};

// Four consecutive elements of a row, from a multiple of four.
__device__ __forceinline__ void put(const Planes& o, int z, int row, int k, f32x4 v) {
  uint16_t* to = o.at(z, row, k);
  const float s = power(o.e);
  uint16_t q[4][2];
#pragma unroll
  for (int e = 0; e < 4; ++e) cut<2>(v[e] * s, q[e]);
#pragma unroll
  for (int p = 0; p < 2; ++p)
    *reinterpret_cast<ushort4*>(to + p * 32) = make_ushort4(q[0][p], q[1][p], q[2][p], q[3][p]);
}
// The same four values as one element of four consecutive rows.
__device__ __forceinline__ void put_across(const Planes& o, int z, int row, int k, int rows, f32x4 v) {
  uint16_t* to = o.at(z, row, k);
  const float s = power(o.e);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (row + e >= rows) continue;
    uint16_t q[2];
    cut<2>(v[e] * s, q);
    to[(long)e * o.ld * 2] = q[0];
    to[(long)e * o.ld * 2 + 32] = q[1];
  }
}

// G -> X: 64 x 64 values a work group.
__global__ __launch_bounds__(256) void k_update_planes(const void* __restrict__ g, UpdateArgs a, int r, int c,
                                                       int across, const double* __restrict__ norms, Planes x) {
  __shared__ float tile[64][65];
  __shared__ double sums[4];
  double s = norms[blockIdx.z * kNormParts + threadIdx.x];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  const double inv = 1.0 / (__builtin_sqrt(sums[0] + sums[1] + sums[2] + sums[3]) + (double)a.eps);
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;   // of X
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 8
  for (int i = 0; i < 16; ++i) {
    // lanes along the rows of G
    const int q = wave + i * 4, rr = across ? r0 + lane : r0 + q, cc = across ? c0 + q : c0 + lane;
    float v = 0;
    if (rr < r && cc < c) {
      const long at = blockIdx.z * a.g_batch + (across ? (long)cc * a.g_stride + rr : (long)rr * a.g_stride + cc);
      v = (float)((double)value(g, at, a.g_bf16) * inv);
    }
    if (across) tile[lane][q] = v;
    else tile[q][lane] = v;
  }
  __syncthreads();
  const float unit = power(x.e);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (threadIdx.x >> 3) + i * 32, k = (threadIdx.x & 7) * 8;
    if (r0 + row >= r) continue;
    __attribute__((aligned(16))) uint16_t out[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t h[2];
      cut<2>(tile[row][k + e] * unit, h);
      out[0][e] = h[0];
      out[1][e] = h[1];
    }
    uint16_t* to = x.at(blockIdx.z, r0 + row, c0 + k);
    *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(out[0]);
    *reinterpret_cast<uint4*>(to + 32) = *reinterpret_cast<const uint4*>(out[1]);
  }
}

// What becomes of the products.  kGram: A.  kPoly: P.  kNext: X.  kLast: the result.
enum Kind { kGram, kPoly, kNext, kLast };
struct Result {
  Planes out;             // of A, P or X
  Planes gram;            // kPoly: A
  int r, c;               // sides of X
  int e;                  // exponents of the two operands, added
  float a, b, c2, scale;
  int across, bf16;       // kLast
  void* o;
  long o_batch, o_stride;
};

// Four values D[m .. m + 3][n] of a product of matrix z: elements m of the result's row n.
// kGram, kPoly: `mirror` writes element n of rows m .. m + 3 as well.  Elements behind the matrix, up to
// whole lines, become zeros: the next product multiplies them.
template <Kind KIND>
__device__ __forceinline__ void finish(const Result& s, int z, int m, int n, f32x4 v, bool mirror) {
  const float unit = power(-s.e);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= unit;
  const int km = KIND <= kPoly ? s.r : s.c;   // rows of the first operand
  if constexpr (KIND == kPoly) {
    if (n < s.r && m < s.gram.ld) {
      const uint16_t* at = s.gram.at(z, n, m);
      const ushort4 h = *reinterpret_cast<const ushort4*>(at), l = *reinterpret_cast<const ushort4*>(at + 32);
      const float one = power(-s.gram.e);
      const float old[4] = {f16_value(h.x) + f16_value(l.x), f16_value(h.y) + f16_value(l.y),
                            f16_value(h.z) + f16_value(l.z), f16_value(h.w) + f16_value(l.w)};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = __builtin_fmaf(s.c2, v[e], s.b * (old[e] * one)) + (m + e == n ? s.a : 0.f);
    }
  }
  if constexpr (KIND == kLast) {
    if (n >= s.r) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (m + e >= s.c) continue;
      const long at = z * s.o_batch + (s.across ? (long)(m + e) * s.o_stride + n : (long)n * s.o_stride + m + e);
      if (s.bf16) static_cast<uint16_t*>(s.o)[at] = bf16_bits(s.scale * v[e]);
      else static_cast<float*>(s.o)[at] = s.scale * v[e];
    }
  } else {
    f32x4 k = v;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (m + e >= km) k[e] = 0;
    if (n < s.r && m < s.out.ld) put(s.out, z, n, m, k);
    // zeros behind a row of the mirror image come from the tile that holds them unmirrored
    if (KIND <= kPoly && mirror && n < s.r) put_across(s.out, z, m, n, s.r, v);
  }
}

// Tile of a symmetric result: the i-th with its rows' tile not behind its columns'.
__device__ __forceinline__ void triangle(int i, int& m, int& n) {
  m = (int)((__builtin_sqrtf(8.f * i + 1.f) - 1.f) * 0.5f);
  while ((m + 1) * (m + 2) / 2 <= i) ++m;
  while (m * (m + 1) / 2 > i) --m;
  n = i - m * (m + 1) / 2;
}

// Products of many tiles.  blockIdx.x: matrix and tile (`tiles` a matrix), .y: range of k.  With several
// ranges their fp32 sums go to `parts` [range][matrix][n][m], for k_update_join.
template <class T, Kind KIND>
__global__ __launch_bounds__(T::THREADS) void k_update_product(Operand x, Operand y, int k, int per, int tiles,
                                                               int tiles_m, Result s, float* __restrict__ parts,
                                                               long part, int part_ld) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int at = place_of_group(blockIdx.x, gridDim.x), z = at / tiles;
  int tm, tn;
  if constexpr (KIND <= kPoly) triangle(at - z * tiles, tm, tn);
  else tile_at(at - z * tiles, tiles_m, tiles / tiles_m, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  const int k0 = blockIdx.y * per, k1 = k0 + per < k ? k0 + per : k;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(x, y, z, m0, n0, k0, k1, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int n = n0 + (wn * T::TN + j) * 16 + (lane & 15);
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      const int m = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4;
      if (parts) {
        if (n < s.r && m < part_ld)
          *reinterpret_cast<f32x4*>(parts + blockIdx.y * part + ((long)z * s.r + n) * part_ld + m) = acc[i][j];
      } else {
        finish<KIND>(s, z, m, n, acc[i][j], tm != tn);
      }
    }
  }
}

// Sums of the ranges of a symmetric product's k, 32 x 32 a work group.
template <Kind KIND>
__global__ __launch_bounds__(256) void k_update_join(const float* __restrict__ parts, int count, long part,
                                                     int part_ld, Result s) {
  int tm, tn;
  triangle(blockIdx.x, tm, tn);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = tn * 32 + (wave >> 1) * 16 + (lane & 15), m = tm * 32 + (wave & 1) * 16 + (lane >> 4) * 4;
  f32x4 v = {0, 0, 0, 0};
  if (n < s.r) {
    const float* from = parts + ((long)blockIdx.y * s.r + n) * part_ld + m;
#pragma unroll 4
    for (int q = 0; q < count; ++q) v += *reinterpret_cast<const f32x4*>(from + q * part);
  }
  finish<KIND>(s, blockIdx.y, m, n, v, tm != tn);
}

// The symmetric products of few rows.
template <Kind KIND, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_update_few(Operand x, int k, int tiles, Result s) {
  typedef Few<2, WAVES> T;
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int at = place_of_group(blockIdx.x, gridDim.x), z = at / tiles;
  int tm, tn;
  triangle(at - z * tiles, tm, tn);
  f32x4 acc[1][1] = {};
  multiply<T>(x, x, z, tm * 32, tn * 32, 0, k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (wave >= 4) return;
  finish<KIND>(s, z, tm * 32 + (wave & 1) * 16 + (lane >> 4) * 4, tn * 32 + (wave >> 1) * 16 + (lane & 15), acc[0][0],
               tm != tn);
}

// Tiles of products; AX: k across the rows of the first operand (X in P X).
template <bool AX>
struct Tiles {
  typedef Tile<256, 256, 2, 4, 2, 2, AX> Big;
  typedef Tile<128, 128, 2, 2, 2, 2, AX> Mid;
  typedef Tile<64, 64, 2, 2, 2, 2, AX> Small;
  typedef Tile<64, 64, 2, 2, 2, 4, AX> Deep;   // where two work groups a compute unit are all there are
};

template <Kind KIND>
void product(const UpdateLayout& l, int batch, const Operand& x, const Operand& y, int k, const Result& s,
             float* parts, hipStream_t st) {
  if constexpr (KIND <= kPoly) {
    if (few(l, batch, k)) {
      // eight waves where four would have more than four lines of k each
      const int tm = half_of(tiles_of(l.r, 32));
      const dim3 grid(tm * batch);
      if (k > 32 * 4 * 4) wino_launch((k_update_few<KIND, 8>), grid, dim3(512), st, x, k, tm, s);
      else wino_launch((k_update_few<KIND, 4>), grid, dim3(256), st, x, k, tm, s);
      return;
    }
    const auto go = [&](auto tile) {
      typedef decltype(tile) T;
      const int tiles = half_of(tiles_of(l.r, T::BM)), splits = KIND == kGram ? l.splits : 1;
      const int per = (int)up((k + splits - 1) / splits, 32);
      const long part = (long)batch * l.r * l.rp;
      wino_launch((k_update_product<T, KIND>), dim3(tiles * batch, splits), dim3(T::THREADS), st, x, y, k, per,
                  tiles, 0, s, splits > 1 ? parts : nullptr, part, l.rp);
      if (splits > 1)
        wino_launch((k_update_join<KIND>), dim3(half_of(tiles_of(l.rp, 32)), batch), dim3(256), st,
                    (const float*)parts, splits, part, l.rp, s);
    };
    if (l.side == 128 && KIND == kGram) go(Tiles<false>::Mid{});
    else if ((long)half_of(tiles_of(l.r, 64)) * batch * (KIND == kGram ? l.splits : 1) <= 512) go(Tiles<false>::Deep{});
    else go(Tiles<false>::Small{});
  } else {
    const auto go = [&](auto tile) {
      typedef decltype(tile) T;
      const int tm = tiles_of(l.c, T::BM), tn = tiles_of(l.r, T::BN);
      wino_launch((k_update_product<T, KIND>), dim3(tm * tn * batch), dim3(T::THREADS), st, x, y, k, k, tm * tn, tm,
                  s, (float*)nullptr, 0L, 0);
    };
    const int side = next_side(l, batch);
    if (side == 256) go(Tiles<true>::Big{});
    else if (side == 128) go(Tiles<true>::Mid{});
    else if ((long)tiles_of(l.c, 64) * tiles_of(l.r, 64) * batch <= 512) go(Tiles<true>::Deep{});
    else go(Tiles<true>::Small{});
  }
}

// Exponent that brings magnitudes up to `most` to 2^15 or below.
int exponent(double most) {
  int e = 0;
  if (!(most > 1e-30)) most = 1e-30;
  if (!(most < 1e30)) most = 1e30;
  std::frexp(most, &e);
  return 15 - e;
}

}  // namespace

hipError_t launch_update(const UpdateArgs& a, const void* g, void* o, char* ws, hipStream_t st) {
  const UpdateLayout l = update_layout(a);
  const int across = a.rows > a.cols;
  double* norms = reinterpret_cast<double*>(ws + l.norms);
  wino_launch(k_update_norm, dim3(kNormParts, a.batch), dim3(256), st, g, a, norms);
  const auto planes = [&](size_t at, int ld, int e) {
    const long items = (long)l.r * ld * 2;
    return Planes{reinterpret_cast<uint16_t*>(ws + at), items, ld, e};
  };
  const auto operand = [&](const Planes& p) { return Operand{p.p, p.ld * 2L, p.batch, l.r, p.ld}; };
  // largest singular value that X can have
  double s = 1;
  Planes x = planes(l.x, l.cp, exponent(s));
  wino_launch(k_update_planes, dim3(l.cp / 64, l.rp / 64, a.batch), dim3(256), st, g, a, l.r, l.c, across,
              (const double*)norms, x);
  float* parts = reinterpret_cast<float*>(ws + l.parts);
  const int rk = (int)up(l.r, 32);
  for (int i = 0; i < a.steps; ++i) {
    // largest |p(t)|, p(t) = a + b t + c t^2 on [0, s^2], and largest s |p(s^2)|: at the ends or where
    // the derivative vanishes
    const double A = a.a, B = a.b, C = a.c, end = s * s;
    double most_p = std::fmax(std::fabs(A), std::fabs(A + B * end + C * end * end)), most_x = 0;
    const auto at = [&](double t) {
      if (!(t >= 0 && t <= end)) return;
      const double p = std::fabs(A + B * t + C * t * t);
      most_p = std::fmax(most_p, p);
      most_x = std::fmax(most_x, std::sqrt(t) * p);
    };
    at(end);
    if (C != 0) {
      at(-B / (2 * C));
      const double root = std::sqrt(std::fmax(0.0, 9 * B * B - 20 * A * C));
      at((-3 * B + root) / (10 * C));
      at((-3 * B - root) / (10 * C));
    } else if (B != 0) {
      at(-A / (3 * B));
    }
    const Planes gram = planes(l.gram, l.rp, exponent(end)), poly = planes(l.poly, l.rp, exponent(most_p));
    Result q{};
    q.r = l.r, q.c = l.c, q.a = a.a, q.b = a.b, q.c2 = a.c, q.scale = a.scale;
    q.across = across, q.bf16 = a.o_bf16, q.o = o, q.o_batch = a.o_batch, q.o_stride = a.o_stride;
    q.out = gram, q.e = 2 * x.e;
    product<kGram>(l, a.batch, operand(x), operand(x), (int)up(l.c, 32), q, parts, st);
    q.out = poly, q.gram = gram, q.e = 2 * gram.e;
    product<kPoly>(l, a.batch, operand(gram), operand(gram), rk, q, parts, st);
    // Room for the products' roundings, and no more: the usual coefficients keep [0, 1.26] within
    // itself, from 1.27 on every step would enlarge it.
    s = 1.0001 * most_x;
    const Planes next = planes(i & 1 ? l.x : l.x2, l.cp, exponent(s));
    q.out = next, q.e = x.e + poly.e;
    if (i + 1 < a.steps) product<kNext>(l, a.batch, operand(x), operand(poly), rk, q, parts, st);
    else product<kLast>(l, a.batch, operand(x), operand(poly), rk, q, parts, st);
    x = next;
  }
  return hipGetLastError();
}

}  // namespace wino
