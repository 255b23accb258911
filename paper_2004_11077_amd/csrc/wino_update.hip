// Orthogonalising a weight gradient by Newton-Schulz products:
//
//   X = G / (|G|_F + eps);  `steps` times  A = X X^T,  X <- a X + (b A + c A A) X;  O = scale X
//
// on the smaller side's products (a taller matrix is taken across).  Three products a step, each with
// its k contiguous in both operands (wino_products.hpp): A from X, the polynomial a I + b A + c A A from
// A, which is symmetric, and the new X from the polynomial and X across.  Every product therefore leaves
// its result cut into planes, the new X both ways.  The step multiplies small singular values by a, an
// error of an early step with them: fp32 results take three planes (24 bits), bf16 results two (16
// bits, which after the amplification by 3.4^4 of the usual coefficients still lies below their
// rounding).
#include "wino_products.hpp"
#include "wino_train.hpp"

namespace wino {
namespace {

using namespace prod;

constexpr int kNormParts = 64;

__device__ __forceinline__ float value(const void* p, long i, int bf16) {
  return bf16 ? bf16_value(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// Sums of squares of a matrix in 64 bits: no square over- or underflows.
__global__ __launch_bounds__(256) void k_update_norm(const void* __restrict__ g, UpdateArgs a,
                                                     double* __restrict__ norms) {
  __shared__ double lds[4];
  const long base = blockIdx.y * a.g_batch, items = (long)a.rows * a.cols;
  double s = 0;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < items; i += kNormParts * 256) {
    const long r = i / a.cols;
    const double v = value(g, base + r * a.g_stride + (i - r * a.cols), a.g_bf16);
    s += v * v;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) norms[blockIdx.y * kNormParts + blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}

// Planes of X, both ways.
struct Planes {
  uint16_t *x, *xt;
  long x_ld, x_plane, x_batch, xt_ld, xt_plane, xt_batch;
};

// G -> X: 64 x 64 values a work group.
template <int NP>
__global__ __launch_bounds__(256) void k_update_planes(const void* __restrict__ g, UpdateArgs a, int r, int c,
                                                       int across, const double* __restrict__ norms,
                                                       Planes p) {
  __shared__ float tile[64][65];
  __shared__ double total;
  if (threadIdx.x < 64) {
    double s = norms[blockIdx.z * kNormParts + threadIdx.x];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
    if (threadIdx.x == 0) total = s;
  }
  __syncthreads();
  const double inv = 1.0 / (__builtin_sqrt(total) + (double)a.eps);
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;   // of X
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll 4
  for (int i = 0; i < 16; ++i) {
    // lanes along the rows of G
    const int q = y + i * 4, rr = across ? r0 + x : r0 + q, cc = across ? c0 + q : c0 + x;
    float v = 0;
    if (rr < r && cc < c) {
      const long at = blockIdx.z * a.g_batch + (across ? (long)cc * a.g_stride + rr : (long)rr * a.g_stride + cc);
      v = (float)((double)value(g, at, a.g_bf16) * inv);
    }
    if (across) tile[x][q] = v;
    else tile[q][x] = v;
  }
  __syncthreads();
  const int row = threadIdx.x >> 2, eight = (threadIdx.x & 3) * 16;
#pragma unroll
  for (int way = 0; way < 2; ++way) {
    const int first = way ? c0 : r0, rows = way ? c : r;
    if (first + row >= rows) continue;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      __attribute__((aligned(16))) uint16_t out[NP][8];
      const int at = eight + half * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint16_t q[NP];
        cut<NP>(way ? tile[at + e][row] : tile[row][at + e], q);
#pragma unroll
        for (int n = 0; n < NP; ++n) out[n][e] = q[n];
      }
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        uint16_t* to = way ? p.xt + n * p.xt_plane + blockIdx.z * p.xt_batch + (long)(c0 + row) * p.xt_ld + r0 + at
                           : p.x + n * p.x_plane + blockIdx.z * p.x_batch + (long)(r0 + row) * p.x_ld + c0 + at;
        *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(out[n]);
      }
    }
  }
}

// Four values of a row of planes, from element m.
template <int NP>
__device__ __forceinline__ void put(uint16_t* to, long plane, const float (&v)[4]) {
  uint16_t q[4][NP];
#pragma unroll
  for (int e = 0; e < 4; ++e) cut<NP>(v[e], q[e]);
#pragma unroll
  for (int p = 0; p < NP; ++p)
    *reinterpret_cast<ushort4*>(to + p * plane) = make_ushort4(q[0][p], q[1][p], q[2][p], q[3][p]);
}

// One symmetric result [r][rp] on planes.
struct Symmetric {
  uint16_t* out;
  long ld, plane, batch;
  int r;
};

// poly = 0: A = X X^T.  poly = 1: a I + b A + c A A from A.
template <class T, bool POLY>
__global__ __launch_bounds__(T::THREADS) void k_update_symmetric(Operand x, Symmetric s, int k, int tiles,
                                                                 float a, float b, float c) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * T::STAGE];
  const int m0 = blockIdx.x % tiles * T::BM, n0 = blockIdx.x / tiles * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(x, x, blockIdx.z, m0, n0, 0, k, k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int n = n0 + (wn * T::TN + j) * 16 + (lane & 15);
    if (n >= s.r) continue;
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      const int m = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4;
      if (m >= s.ld) continue;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e];
      if constexpr (POLY) {
        float old[4] = {};
#pragma unroll
        for (int p = T::NP - 1; p >= 0; --p) {
          const ushort4 q = *reinterpret_cast<const ushort4*>(x.p + p * x.plane + blockIdx.z * x.batch + (long)n * x.ld + m);
          old[0] += bf16_value(q.x), old[1] += bf16_value(q.y), old[2] += bf16_value(q.z), old[3] += bf16_value(q.w);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(c, v[e], b * old[e]) + (m + e == n ? a : 0.f);
      }
      put<T::NP>(s.out + blockIdx.z * s.batch + (long)n * s.ld + m, s.plane, v);
    }
  }
}

// New X, both ways; the last step leaves the result instead.
template <class T, bool LAST>
__global__ __launch_bounds__(T::THREADS) void k_update_next(Operand xt, Operand poly, Planes p, int k,
                                                            int tiles_m, UpdateArgs u, int across, void* o) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * T::STAGE];
  const int m0 = blockIdx.x % tiles_m * T::BM, n0 = blockIdx.x / tiles_m * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(xt, poly, blockIdx.z, m0, n0, 0, k, k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int n = n0 + (wn * T::TN + j) * 16 + (lane & 15);   // row of X
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      const int m = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4;   // column of X
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e];
      if constexpr (LAST) {
        if (n >= poly.rows) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (m + e >= xt.rows) continue;
          const long at = blockIdx.z * u.o_batch + (across ? (long)(m + e) * u.o_stride + n : (long)n * u.o_stride + m + e);
          if (u.o_bf16) static_cast<uint16_t*>(o)[at] = bf16_bits(u.scale * v[e]);
          else static_cast<float*>(o)[at] = u.scale * v[e];
        }
      } else {
        if (n < poly.rows && m < p.x_ld)
          put<T::NP>(p.x + blockIdx.z * p.x_batch + (long)n * p.x_ld + m, p.x_plane, v);
        if (n < p.xt_ld)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (m + e >= xt.rows) continue;
            uint16_t q[T::NP];
            cut<T::NP>(v[e], q);
#pragma unroll
            for (int s = 0; s < T::NP; ++s)
              p.xt[s * p.xt_plane + blockIdx.z * p.xt_batch + (long)(m + e) * p.xt_ld + n] = q[s];
          }
      }
    }
  }
}

template <int NP>
hipError_t update(const UpdateArgs& a, const void* g, void* o, char* ws, hipStream_t st) {
  typedef Tile<128, 128, 2, 2, NP> T;
  const UpdateLayout l = update_layout(a);
  const int across = a.rows > a.cols;
  double* norms = reinterpret_cast<double*>(ws + l.norms);
  wino_launch(k_update_norm, dim3(kNormParts, a.batch), dim3(256), st, g, a, norms);
  const long xb = (long)l.r * l.cp, tb = (long)l.c * l.rp, sb = (long)l.r * l.rp;
  Planes p[2];
  for (int i = 0; i < 2; ++i)
    p[i] = Planes{reinterpret_cast<uint16_t*>(ws + (i ? l.x2 : l.x)), reinterpret_cast<uint16_t*>(ws + (i ? l.xt2 : l.xt)),
                  l.cp, xb * a.batch, xb, l.rp, tb * a.batch, tb};
  uint16_t* gram = reinterpret_cast<uint16_t*>(ws + l.gram);
  uint16_t* poly = reinterpret_cast<uint16_t*>(ws + l.poly);
  wino_launch((k_update_planes<NP>), dim3(l.cp / 64, l.rp / 64, a.batch), dim3(256), st, g, a, l.r, l.c, across,
              (const double*)norms, p[0]);
  const int tr = (l.rp + T::BM - 1) / T::BM, tc = (l.cp + T::BM - 1) / T::BM;
  const Symmetric sg{gram, l.rp, sb * a.batch, sb, l.r}, sp{poly, l.rp, sb * a.batch, sb, l.r};
  const Operand og{gram, l.rp, sb * a.batch, sb, l.r}, op{poly, l.rp, sb * a.batch, sb, l.r};
  for (int s = 0; s < a.steps; ++s) {
    const Planes& from = p[s & 1];
    const Operand ox{from.x, l.cp, xb * a.batch, xb, l.r}, ot{from.xt, l.rp, tb * a.batch, tb, l.c};
    wino_launch((k_update_symmetric<T, false>), dim3(tr * tr, 1, a.batch), dim3(T::THREADS), st, ox, sg, l.cp, tr, a.a,
                a.b, a.c);
    wino_launch((k_update_symmetric<T, true>), dim3(tr * tr, 1, a.batch), dim3(T::THREADS), st, og, sp, l.rp, tr, a.a,
                a.b, a.c);
    if (s + 1 < a.steps)
      wino_launch((k_update_next<T, false>), dim3(tc * tr, 1, a.batch), dim3(T::THREADS), st, ot, op, p[~s & 1], l.rp,
                  tc, a, across, o);
    else
      wino_launch((k_update_next<T, true>), dim3(tc * tr, 1, a.batch), dim3(T::THREADS), st, ot, op, p[~s & 1], l.rp,
                  tc, a, across, o);
  }
  return hipGetLastError();
}

}  // namespace

UpdateLayout update_layout(const UpdateArgs& a) {
  UpdateLayout l{};
  l.planes = a.o_bf16 ? 2 : 3;
  l.r = a.rows < a.cols ? a.rows : a.cols;
  l.c = a.rows < a.cols ? a.cols : a.rows;
  l.rp = (int)up(l.r, 64);
  l.cp = (int)up(l.c, 64);
  size_t at = 0;
  const auto take = [&](size_t bytes) { const size_t was = at; at += up(bytes, 256); return was; };
  const size_t item = 2 * (size_t)l.planes * a.batch;
  l.norms = take(sizeof(double) * kNormParts * a.batch);
  l.x = take(item * l.r * l.cp);
  l.xt = take(item * l.c * l.rp);
  l.x2 = take(item * l.r * l.cp);
  l.xt2 = take(item * l.c * l.rp);
  l.gram = take(item * l.r * l.rp);
  l.poly = take(item * l.r * l.rp);
  l.bytes = at ? at : 256;
  return l;
}

hipError_t launch_update(const UpdateArgs& a, const void* g, void* o, char* ws, hipStream_t st) {
  return a.o_bf16 ? update<2>(a, g, o, ws, st) : update<3>(a, g, o, ws, st);
}

}  // namespace wino
