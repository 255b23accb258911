// Layer norm over the channels of a row (a pixel of an NHWC tensor), forward and backward.
//
//   mu = sum x / C,  v = sum (x - mu)^2 / C,  s = 1 / sqrt(v + eps),  y = (x - mu) s gamma + beta
//   xh = (x - mu) s, g = dy gamma:  dx = s (g - mean(g) - xh mean(g xh)),
//   dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//
// What bounds it is memory: each tensor passes once.  8192 x 4096 fp32, 268 MB: 50.4 us, 5.3 TB/s (the copy of a
// large tensor reaches 4.86), bf16, 134 MB: 32.5 us; backward 16384 x 256 fp32, 50.4 MB: 13.7 us, 3.7 TB/s, of
// which 3.4 to 3.8 us are the second launch that joins the columns' sums; 8192 x 4096 bf16, 201 MB: 53.7 us, 3.7
// TB/s.  Codes wait for their 64-bit arithmetic as well: 131072 x 64 fp32 to codes, 42.5 MB, takes 13.4 us, to bf16,
// 50 MB, 11.7, to fp32, 67 MB, 13.7.  64 x 16: 2.2 us, a launch.
//
// A row is read once and stays in registers between its sums: LANES lanes hold it, NV vectors of VEC
// values each.  The variance is the sum of squared differences from the mean, never a difference of
// large sums.  Everything is fp32, but 64 bits where int8 codes come out: a code then equals the
// formula's, also next to a border between two codes, where 32 bits decide one value in 10^6 the
// other way.
#include "wino_kernels.hpp"
#include "wino_train.hpp"

namespace wino {
namespace {

constexpr int kF32 = 0, kBf16 = 1, kI8 = 2;

template <class T, int N>
using vec_of = __attribute__((ext_vector_type(N))) T;

struct bf16_t { uint16_t bits; };
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __builtin_bit_cast(float, (uint32_t)v.bits << 16); }

// VEC values from p (aligned to all of them when VEC > 1).
template <int VEC>
__device__ __forceinline__ void load(const float* p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = *p;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const vec_of<float, 4> q = *reinterpret_cast<const vec_of<float, 4>*>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = q[e];
    }
  }
}
template <int VEC>
__device__ __forceinline__ void load(const bf16_t* p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = widen(*p);
  } else {
    typedef vec_of<uint16_t, VEC> V;
    const V q = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = widen(bf16_t{q[e]});
  }
}
template <int VEC>
__device__ __forceinline__ void store(float* p, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    *p = v[0];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4)
      *reinterpret_cast<vec_of<float, 4>*>(p + i) = vec_of<float, 4>{v[i], v[i + 1], v[i + 2], v[i + 3]};
  }
}
template <int VEC>
__device__ __forceinline__ void store(bf16_t* p, const float (&v)[VEC]) {
  vec_of<uint16_t, VEC> q;
#pragma unroll
  for (int e = 0; e < VEC; ++e) q[e] = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
  if constexpr (VEC == 1) p->bits = q[0];
  else *reinterpret_cast<vec_of<uint16_t, VEC>*>(p) = q;
}
template <int VEC>
__device__ __forceinline__ void store(int8_t* p, const int (&v)[VEC]) {
  vec_of<int8_t, VEC> q;
#pragma unroll
  for (int e = 0; e < VEC; ++e) q[e] = (int8_t)v[e];
  if constexpr (VEC == 1) *p = q[0];
  else *reinterpret_cast<vec_of<int8_t, VEC>*>(p) = q;
}

// Sum over the LANES lanes of a row; `lds`: one value per wave where a row spans several.  Every
// thread of the work group calls it.  The order is fixed.
template <int LANES, class F>
__device__ __forceinline__ F sum_lanes(F v, F* lds) {
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v += __shfl_xor(v, d, 64);
  if constexpr (LANES > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) v += lds[w];
  }
  return v;
}

template <int LANES>
constexpr int kThreads = LANES > 256 ? LANES : 256;
// Backward pass: sixteen waves a work group where their sums of columns fit 32 KiB of LDS.
template <int LANES, int PER>
constexpr int kBackThreads = LANES > 256 ? LANES : PER <= 8 ? 1024 : PER <= 16 ? 512 : 256;

// Both sums over the LANES lanes of a row; `lds`: a float2 per wave, another buffer than in the call
// before, so that one barrier is enough.
template <int LANES>
__device__ __forceinline__ void sum_pair(float& a, float& b, float2* lds) {
#pragma unroll
  for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) a += __shfl_xor(a, d, 64), b += __shfl_xor(b, d, 64);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    const float2* mine = lds + threadIdx.x / LANES * (LANES / 64);
    a = mine[0].x, b = mine[0].y;
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) a += mine[w].x, b += mine[w].y;
  }
}

// The code of a quotient; F is double exactly where these come out.
__device__ __forceinline__ int code_of(double q) {
  q = __builtin_rint(q);
  q = q > 127 ? 127 : q < -127 ? -127 : q;
  return (int)q;   // a NaN gives 0
}
// Codes of VEC values y for steps of s: rint(y / s) with the correctly rounded quotient, so that what lies on the
// border between two codes is rounded as the formula rounds it.  The product with 1 / s may be a last place off
// either way (it moves 7617 of the borders of s = n 2^-14, odd n below 2000), which matters next to a border
// alone: there its residual, exact but for a last place of its own, puts it right.
template <int VEC>
__device__ __forceinline__ void codes_of(const double (&y)[VEC], double s, double inv_s, int (&out)[VEC]) {
  bool near = false;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const double q = y[e] * inv_s;
    near |= __builtin_fabs(q - __builtin_rint(q)) > 0.49999;   // not so for infinities and NaN
    out[e] = code_of(q);
  }
  if (near)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const double q = y[e] * inv_s;
      if (__builtin_fabs(q) < 256) out[e] = code_of(__builtin_fma(__builtin_fma(-q, s, y[e]), inv_s, q));
    }
}

// A row's mean, the correctly rounded quotient where the product with 1 / channels may be a last place off: a row of
// one value whose sum is exact has that value as its mean and nothing left beside it, neither to be divided by the
// root of eps nor to move a code off its border.
template <class F>
__device__ __forceinline__ F mean_of(F sum, const NormArgs& a) {
  const F q = sum * (F)a.inv_c, left = __builtin_elementwise_fma(-q, (F)a.channels, sum);
  return left == left ? __builtin_elementwise_fma(left, (F)a.inv_c, q) : q;   // an infinite sum leaves a NaN
}

// 1 / sqrt(v).  64 bits: the instruction's 26 bits and two steps of r <- r (3 - v r r) / 2; of zero (a row of one value
// and no eps) infinity, from which a step would make a NaN.
__device__ __forceinline__ float inverse_root(float v) { return 1.f / __builtin_sqrtf(v); }
__device__ __forceinline__ double inverse_root(double v) {
  double r = __builtin_amdgcn_rsq(v);
#pragma unroll
  for (int i = 0; i < 2; ++i) r = r * __builtin_fma(-0.5 * v * r, r, 1.5);
  return v == 0 ? __builtin_inf() : r;
}

template <class TI, class F, int LANES, int VEC, int NV>
__global__ __launch_bounds__(kThreads<LANES>) void k_norm(NormArgs a, const TI* __restrict__ x,
                                                          const float* __restrict__ gamma,
                                                          const float* __restrict__ beta,
                                                          void* __restrict__ y, float* __restrict__ mean,
                                                          float* __restrict__ rstd) {
  __shared__ F lds[16];
  constexpr int ROWS = kThreads<LANES> / LANES;
  const int lane = threadIdx.x % LANES;
  const int C = a.channels;
  for (long first = (long)blockIdx.x * ROWS; first < a.rows; first += (long)gridDim.x * ROWS) {
  const long row = first + threadIdx.x / LANES;
  const bool live = row < a.rows;
  const TI* px = x + (live ? row : 0) * a.x_stride;
  float v[NV][VEC];
  F sum = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LANES + lane) * VEC;
    if (c < C) load<VEC>(px + c, v[i]);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum += (F)v[i][e];
  }
  const F mu = mean_of(sum_lanes<LANES>(sum, lds), a);
  F sq = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const bool in = (i * LANES + lane) * VEC < C;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const F d = in ? (F)v[i][e] - mu : 0;
      sq = __builtin_elementwise_fma(d, d, sq);
    }
  }
  const F var = sum_lanes<LANES>(sq, lds) * (F)a.inv_c;
  const F s = inverse_root(var + (F)a.eps);
  if (!live) continue;   // no other lane of this row's work group waits for these
  if (lane == 0) {
    if (mean) mean[row] = (float)mu;
    if (rstd) rstd[row] = (float)s;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LANES + lane) * VEC;
    if (c >= C) continue;
    float ga[VEC], be[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) ga[e] = 1, be[e] = 0;
    if (gamma) load<VEC>(gamma + c, ga);
    if (beta) load<VEC>(beta + c, be);
    const long at = row * a.y_stride + c;
    if constexpr (sizeof(F) == 8) {
      int q[VEC];
      constexpr int AT_ONCE = VEC < 2 ? VEC : 2;   // fewer registers (131072 x 64 of bf16: 17.8 us, eight at once 19.0)
#pragma unroll
      for (int b = 0; b < VEC; b += AT_ONCE) {
        F o[AT_ONCE];
        int p[AT_ONCE];
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) o[e] = ((F)v[i][b + e] - mu) * s * (F)ga[b + e] + (F)be[b + e];
        codes_of<AT_ONCE>(o, a.s, a.inv_s, p);
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) q[b + e] = p[e];
      }
      store<VEC>(static_cast<int8_t*>(y) + at, q);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] = __builtin_fmaf((v[i][e] - mu) * s, ga[e], be[e]);
      if (a.y_type == kF32) store<VEC>(static_cast<float*>(y) + at, v[i]);
      else store<VEC>(static_cast<bf16_t*>(y) + at, v[i]);
    }
  }
  }
}

// Rows too long for registers: a work group reads its row three times, from the cache after the first.
template <class TI, class F>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a, const TI* __restrict__ x,
                                                    const float* __restrict__ gamma,
                                                    const float* __restrict__ beta, void* __restrict__ y,
                                                    float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ F lds[16];
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
  const TI* px = x + row * a.x_stride;
  F sum = 0;
  for (int c = threadIdx.x; c < a.channels; c += 1024) sum += (F)widen(px[c]);
  const F mu = mean_of(sum_lanes<1024>(sum, lds), a);
  F sq = 0;
  for (int c = threadIdx.x; c < a.channels; c += 1024) {
    const F d = (F)widen(px[c]) - mu;
    sq = __builtin_elementwise_fma(d, d, sq);
  }
  const F var = sum_lanes<1024>(sq, lds) * (F)a.inv_c;
  const F s = inverse_root(var + (F)a.eps);
  if (threadIdx.x == 0) {
    if (mean) mean[row] = (float)mu;
    if (rstd) rstd[row] = (float)s;
  }
  for (int c = threadIdx.x; c < a.channels; c += 1024) {
    const F ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
    const long at = row * a.y_stride + c;
    const F v = ((F)widen(px[c]) - mu) * s;
    if constexpr (sizeof(F) == 8) {
      const F o[1] = {v * ga + be};
      int q[1];
      codes_of<1>(o, a.s, a.inv_s, q);
      store<1>(static_cast<int8_t*>(y) + at, q);
    } else {
      const float o[1] = {__builtin_fmaf(v, ga, be)};
      if (a.y_type == kF32) store<1>(static_cast<float*>(y) + at, o);
      else store<1>(static_cast<bf16_t*>(y) + at, o);
    }
  }
  }
}

// Values as they lie in memory, widened when they are used: the next row's are under way while this
// one's sums are taken.
template <class T, int VEC>
struct Raw {
  vec_of<T, VEC> v;
  __device__ __forceinline__ float operator[](int e) const { return v[e]; }
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = x;
  }
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC == 1) v[0] = *p;
    else v = *reinterpret_cast<const vec_of<T, VEC>*>(p);
  }
};
template <int VEC>
struct Raw<bf16_t, VEC> {
  vec_of<uint16_t, VEC> v;
  __device__ __forceinline__ float operator[](int e) const { return widen(bf16_t{v[e]}); }
  __device__ __forceinline__ void load(const bf16_t* p) {
    if constexpr (VEC == 1) v[0] = p->bits;
    else v = *reinterpret_cast<const vec_of<uint16_t, VEC>*>(p);
  }
};

// Backward pass.  A work group takes every gridDim-th set of rows; its lanes keep their channels' sums
// of dy xh and dy in registers over all its rows, joins the sets of a work group in LDS and leaves one
// partial sum per work group: no atomics, so the order of the sums is fixed.
template <class TI, class TG, int LANES, int VEC, int NV>
__global__ __launch_bounds__((kBackThreads<LANES, NV * VEC>)) void k_norm_backward(
    NormArgs a, const TG* __restrict__ dy, const TI* __restrict__ x, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, TG* __restrict__ dx,
    float* __restrict__ parts) {
  __shared__ float2 lds[2][16];
  constexpr int THREADS = kBackThreads<LANES, NV * VEC>, ROWS = THREADS / LANES;
  int turn = 0;
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  const int C = a.channels;
  float dg[NV][VEC] = {}, db[NV][VEC] = {};
  const float inv_c = (float)a.inv_c;
  Raw<TI, VEC> nx[NV];
  Raw<TG, VEC> ng[NV];
  float next_mu = 0, next_s = 0;
  const auto fetch = [&](long row) {
    if (row >= a.rows) return;
    next_mu = mean[row], next_s = rstd[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * VEC;
      if (c < C) nx[i].load(x + row * a.x_stride + c), ng[i].load(dy + row * a.dy_stride + c);
    }
  };
  fetch((long)blockIdx.x * ROWS + sub);
  for (long first = (long)blockIdx.x * ROWS; first < a.rows; first += (long)gridDim.x * ROWS) {
    const long row = first + sub;
    const bool live = row < a.rows;
    const float mu = next_mu, s = next_s;
    float vx[NV][VEC], vg[NV][VEC];
    float s1 = 0, s2 = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * VEC;
      const bool in = live && c < C;
      float ga[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) ga[e] = 1;
      if (gamma && c < C) load<VEC>(gamma + c, ga);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = in ? (nx[i][e] - mu) * s : 0.f, d = in ? ng[i][e] : 0.f;
        dg[i][e] = __builtin_fmaf(d, xh, dg[i][e]);
        db[i][e] += d;
        vx[i][e] = xh;
        vg[i][e] = d * ga[e];
        s1 += vg[i][e];
        s2 = __builtin_fmaf(vg[i][e], xh, s2);
      }
    }
    fetch(row + (long)gridDim.x * ROWS);
    sum_pair<LANES>(s1, s2, lds[turn ^= 1]);
    s1 *= inv_c, s2 *= inv_c;
    if (live && dx) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * LANES + lane) * VEC;
        if (c >= C) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) vg[i][e] = s * (vg[i][e] - s1 - vx[i][e] * s2);
        store<VEC>(dx + row * a.dx_stride + c, vg[i]);
      }
    }
  }
  if (!parts) return;
  float* out = parts + (long)blockIdx.x * 2 * C;
  if constexpr (ROWS > 1) {
    __shared__ float join[THREADS * NV * VEC];   // [set of rows][vector][lane][element]
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          join[sub * LANES * NV * VEC + (i * LANES + lane) * VEC + e] = which ? db[i][e] : dg[i][e];
      __syncthreads();
      for (int c = threadIdx.x; c < C; c += THREADS) {
        float v = join[c];
#pragma unroll 4
        for (int q = 1; q < ROWS; ++q) v += join[q * LANES * NV * VEC + c];
        out[which * C + c] = v;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * VEC;
      if (c < C)
#pragma unroll
        for (int e = 0; e < VEC; ++e) out[c + e] = dg[i][e], out[C + c + e] = db[i][e];
    }
  }
}

// Rows too long for registers: dx by one work group a row, and the sums over rows by columns.
template <class TI, class TG>
__global__ __launch_bounds__(1024) void k_norm_backward_long(
    NormArgs a, const TG* __restrict__ dy, const TI* __restrict__ x, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, TG* __restrict__ dx) {
  __shared__ float lds[16], lds2[16];
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
  const TI* px = x + row * a.x_stride;
  const TG* pg = dy + row * a.dy_stride;
  const float mu = mean[row], s = rstd[row], inv_c = (float)a.inv_c;
  float s1 = 0, s2 = 0;
  for (int c = threadIdx.x; c < a.channels; c += 1024) {
    const float g = widen(pg[c]) * (gamma ? gamma[c] : 1.f), xh = (widen(px[c]) - mu) * s;
    s1 += g;
    s2 = __builtin_fmaf(g, xh, s2);
  }
  s1 = sum_lanes<1024>(s1, lds) * inv_c;
  s2 = sum_lanes<1024>(s2, lds2) * inv_c;
  for (int c = threadIdx.x; c < a.channels; c += 1024) {
    const float g = widen(pg[c]) * (gamma ? gamma[c] : 1.f), xh = (widen(px[c]) - mu) * s;
    const float o[1] = {s * (g - s1 - xh * s2)};
    store<1>(dx + row * a.dx_stride + c, o);
  }
  }
}

template <class TI, class TG>
__global__ __launch_bounds__(256) void k_norm_columns_long(NormArgs a, const TG* __restrict__ dy,
                                                           const TI* __restrict__ x,
                                                           const float* __restrict__ mean,
                                                           const float* __restrict__ rstd,
                                                           float* __restrict__ parts) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.channels) return;
  float dg = 0, db = 0;
  for (long row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float d = widen(dy[row * a.dy_stride + c]);
    dg = __builtin_fmaf(d, (widen(x[row * a.x_stride + c]) - mean[row]) * rstd[row], dg);
    db += d;
  }
  float* out = parts + (long)blockIdx.y * 2 * a.channels;
  out[c] = dg;
  out[a.channels + c] = db;
}

// Partial sums [parts][2][C] -> dgamma, dbeta.  16 channels a work group, 64 threads each.
__global__ __launch_bounds__(1024) void k_norm_join(const float* __restrict__ parts, int count, int C,
                                                    float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float lds[64][16];
  const int x = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int c = blockIdx.x * 16 + x;   // of 2 C
  float v = 0;
  if (c < 2 * C)
#pragma unroll 8
    for (int p = g; p < count; p += 64) v += parts[(long)p * 2 * C + c];
  lds[g][x] = v;
  __syncthreads();
  for (int d = 32; d > 0; d /= 2) {
    if (g < d) lds[g][x] += lds[g + d][x];
    __syncthreads();
  }
  if (g == 0 && c < 2 * C) {
    if (c < C) {
      if (dgamma) dgamma[c] = lds[0][x];
    } else if (dbeta) {
      dbeta[c - C] = lds[0][x];
    }
  }
}

// A launch holds fewer than 2^32 threads; what is beyond takes further turns of the kernels' loops.
unsigned grid_of(long blocks) { return (unsigned)(blocks < (1 << 21) ? blocks : 1 << 21); }
bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool at(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Lanes of a row and vectors per lane for `n` vectors, the fewest of both that hold it, so that lanes of
// narrow rows are not idle (64 channels, 16 vectors: four rows a wave) and a wave stays within a row up to
// 256 vectors, whose sums then need no barrier; f(LANES, NV) or
// false where the row is too long.
template <class F>
bool with_shape(long n, F&& f) {
#define SHAPE(L, V) if (n <= L * V) { f(std::integral_constant<int, L>{}, std::integral_constant<int, V>{}); return true; }
  SHAPE(4, 1) SHAPE(16, 1) SHAPE(16, 2) SHAPE(64, 1) SHAPE(64, 2) SHAPE(64, 4) SHAPE(256, 2) SHAPE(256, 4) SHAPE(512, 4)
#undef SHAPE
  return false;
}

template <class TI, class F>
hipError_t norm(const NormArgs& a, const TI* x, const float* gamma, const float* beta, void* y, float* mean,
                float* rstd, hipStream_t st) {
  constexpr int V = 16 / sizeof(TI);
  const int size_y = a.y_type == kF32 ? 4 : a.y_type == kBf16 ? 2 : 1;
  const bool whole = a.channels % V == 0 && a.x_stride % V == 0 && a.y_stride % V == 0 && at16(x) &&
                     at(y, V * size_y > 16 ? 16 : V * size_y) && at16(gamma) && at16(beta);
  const auto go = [&](auto vec) {
    constexpr int VEC = decltype(vec)::value;
    return with_shape(a.channels / VEC, [&](auto lanes, auto nv) {
      constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value, ROWS = kThreads<L> / L;
      wino_launch((k_norm<TI, F, L, VEC, NV>), dim3(grid_of((a.rows + ROWS - 1) / ROWS)),
                  dim3(kThreads<L>), st, a, x, gamma, beta, y, mean, rstd);
    });
  };
  if (!(whole ? go(std::integral_constant<int, V>{}) : go(std::integral_constant<int, 1>{})))
    wino_launch((k_norm_long<TI, F>), dim3(grid_of(a.rows)), dim3(1024), st, a, x, gamma, beta, y, mean, rstd);
  return hipGetLastError();
}

template <class TI, class TG>
hipError_t norm_backward(const NormArgs& a, const TG* dy, const TI* x, const float* gamma, const float* mean,
                         const float* rstd, TG* dx, float* dgamma, float* dbeta, float* parts,
                         hipStream_t st) {
  constexpr int V = 16 / (sizeof(TI) < sizeof(TG) ? sizeof(TI) : sizeof(TG));
  const bool whole = a.channels % V == 0 && a.x_stride % V == 0 && a.dy_stride % V == 0 &&
                     a.dx_stride % V == 0 && at16(x) && at16(dy) && at16(dx) && at16(gamma);
  const int count = norm_parts(a.rows, a.channels);
  const bool sums = dgamma || dbeta;
  float* to = sums ? parts : nullptr;
  const auto go = [&](auto vec) {
    constexpr int VEC = decltype(vec)::value;
    return with_shape(a.channels / VEC, [&](auto lanes, auto nv) {
      constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
      wino_launch((k_norm_backward<TI, TG, L, VEC, NV>), dim3(count), dim3(kBackThreads<L, NV * VEC>), st, a, dy,
                  x, gamma, mean, rstd, dx, to);
    });
  };
  if (!(whole ? go(std::integral_constant<int, V>{}) : go(std::integral_constant<int, 1>{}))) {
    if (dx && a.rows)
      wino_launch((k_norm_backward_long<TI, TG>), dim3(grid_of(a.rows)), dim3(1024), st, a, dy, x, gamma, mean,
                  rstd, dx);
    if (sums)
      wino_launch((k_norm_columns_long<TI, TG>), dim3((a.channels + 255) / 256, count), dim3(256), st, a, dy, x,
                  mean, rstd, to);
  }
  if (sums)
    wino_launch(k_norm_join, dim3((2 * a.channels + 15) / 16), dim3(1024), st, (const float*)parts, count,
                a.channels, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace

int norm_parts(long rows, int channels) {
  // Two work groups a compute unit.  Rows of more than 16384 values go by blocks of 256 columns too (the
  // long form), so that fewer ranges of rows fill the chip, and the partial sums stay within 64 MiB up to
  // 2^23 columns.
  const long most = channels <= 16384 ? 512 : channels < 1 << 23 ? (512L << 14) / channels : 1;
  return (int)(rows < 1 ? 1 : rows < most ? rows : most);
}

hipError_t launch_norm(const NormArgs& a, const void* x, const float* gamma, const float* beta, void* y,
                       float* mean, float* rstd, hipStream_t st) {
  const bool codes = a.y_type == kI8;
  if (a.x_type == kF32)
    return codes ? norm<float, double>(a, (const float*)x, gamma, beta, y, mean, rstd, st)
                 : norm<float, float>(a, (const float*)x, gamma, beta, y, mean, rstd, st);
  return codes ? norm<bf16_t, double>(a, (const bf16_t*)x, gamma, beta, y, mean, rstd, st)
               : norm<bf16_t, float>(a, (const bf16_t*)x, gamma, beta, y, mean, rstd, st);
}

hipError_t launch_norm_backward(const NormArgs& a, const void* dy, const void* x, const float* gamma,
                                const float* mean, const float* rstd, void* dx, float* dgamma,
                                float* dbeta, float* parts, hipStream_t st) {
  const auto go = [&](auto ti, auto tg) {
    typedef decltype(ti) TI;
    typedef decltype(tg) TG;
    return norm_backward<TI, TG>(a, (const TG*)dy, (const TI*)x, gamma, mean, rstd, (TG*)dx, dgamma, dbeta,
                                 parts, st);
  };
  if (a.x_type == kF32) return a.g_type == kF32 ? go(float{}, float{}) : go(float{}, bf16_t{});
  return a.g_type == kF32 ? go(bf16_t{}, float{}) : go(bf16_t{}, bf16_t{});
}

}  // namespace wino
