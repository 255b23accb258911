// Softmax cross entropy of a linear classifier, h W^T + bias, without keeping the logits.
//
//   l = h W^T + b,  lse_t = log sum_v exp(l_tv),  loss_t = lse_t - l_t[target_t]
//   dl_tv = (exp(l_tv - lse_t) - [v = target_t]) dloss_t,  dh = dl W,  dW = dl^T h,  db = sum_t dl
//
// What bounds it: the matrix pipe, 8 T D V operations for a training step of T rows, D features and V
// classes (the logits are computed twice).  T = 4096, D = 2048, V = 65536 in bf16: 4.1 ms, 1.07 PFLOP/s, the
// library's large product at 8192^3 reaching 1.3; 1001 x 515 x 10007 in fp32 on two planes: 270 us, 153
// TFLOP/s of fp32 (459 of the matrix pipe's, tiles that are not full and the planes' copies are the rest).
// Few rows: the weights' passage through memory.  One row of 4096 x 131072 in bf16: 176 us, 6.1 TB/s; a
// training step of 3 x 925 x 75113 in fp32: 324 us, of which 160 read W and write dW.  Small ones: launches,
// 256 x 512 x 10: five in 33 us.
//
// Forward: the logits of a tile leave the matrix instructions in registers and end there as a maximum
// and a sum of exponentials a row; those of all tiles are joined by a second kernel.  Backward: the
// logits are computed again, piece by piece of the classes, and become dl in the workspace, the
// operand of the two products of the piece; h, W and dl enter those with k across their rows
// (wino_products.hpp), so none of them is transposed in memory.
//
// bf16 operands are taken where they lie if their rows are whole pieces of 16 bytes and whole lines, and
// from a padded copy otherwise; dl is rounded to bf16 like the gradients, which then are off by 1.66e-3 to 2.06e-3
// of their 2-norm where rounding the exact ones costs 1.66e-3 (of few rows or small products to two bf16 values, where
// that costs little: one row of two classes was off by 0.004 of the gradient, twice a bf16 result's rounding).  fp32 operands become two
// fp16 planes (22 bits) under one power of two for W and one for h (in the forward pass one a row, so that
// no row's magnitude touches another's lse; of few rows and large W, or few classes and large h, fp32 as it stands, cut between
// LDS and the matrix instructions: W is then read and nothing else); in the backward pass rows that are left out count as
// zeros, whatever they hold, and do not enter the power of two, nor do classes that are masked and no row's target.  dl is kept
// relative to the largest finite |dloss|, by which the products' results are multiplied in fp32: with one weight for all rows, as
// for a mean, the -1 of a target's class stays free of a rounding that would be the same in every row.
#include "wino_products.hpp"
#include "wino_train.hpp"

namespace wino {
namespace {

using namespace prod;
using namespace loss;

constexpr int kDlExponent = 15;    // fp16 planes of dl: |dl| <= 1 relative to the largest |dloss|
constexpr float kInf = __builtin_inff();

// exp(x) for x <= 0 or so by exp2; the argument's rounding is |x| 2^-24, which is most where exp is
// least.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// 2^e with |x| 2^e <= 2^15 for |x| <= most.
__device__ __forceinline__ int exponent_for(float most) {
  const int e = 15 - __builtin_amdgcn_frexp_expf(most);
  return most == 0.f ? 0 : e > 120 ? 120 : e;
}

// Maximum over the threads of a work group; lds: one value per wave.
__device__ __forceinline__ float group_max(float m, float* lds) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
  __syncthreads();
  m = lds[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) m = __builtin_fmaxf(m, lds[w]);
  return m;
}

// What tells the rows that count.
struct Rows {
  const int64_t* target;
  long ignore;
  int rows, classes;
  __device__ __forceinline__ bool kept(int t) const {
    const long c = target[t];
    return c != ignore && c >= 0 && c < classes;
  }
};

__device__ __forceinline__ bool masked(const float* bias, int v) { return bias && bias[v] == -kInf; }

// Largest finite |x| of what blockIdx.x has of a tensor's values, without rows that skip(row) leaves out; m: another
// value of each thread's that counts.  Long rows go by waves, in pieces of 4096, so that a row is asked for once; short
// ones by values.  (300 x 4096 x 60000 with a bias, W's 983 MB: by values 580 us more.)
template <class F>
__device__ __forceinline__ float range_of(const float* x, long ld, int rows, int cols, bool all, F&& skip, float m, float* lds) {
  constexpr int STEP = kRange * 1024, PIECE = 4096;
  const int first = blockIdx.x * 1024 + threadIdx.x;
  const auto take = [&](float v) {
    v = __builtin_fabsf(v);
    m = v < kInf ? __builtin_fmaxf(m, v) : m;
  };
  if (all && ld == cols) {   // one run of values
    const long items = (long)rows * cols;
#pragma unroll 8
    for (long i = first; i < items; i += STEP) take(x[i]);
  } else if (cols >= 128) {
    const int pieces = (cols + PIECE - 1) / PIECE, lane = threadIdx.x & 63;
    const long tasks = (long)rows * pieces;
    for (long task = first >> 6; task < tasks; task += STEP / 64) {
      const int r = (int)(task / pieces), from = (int)(task - (long)r * pieces) * PIECE;
      const int to = cols - from < PIECE ? cols : from + PIECE;
      if (skip(r)) continue;
#pragma unroll 8
      for (int c = from + lane; c < to; c += 64) take(x[r * ld + c]);
    }
  } else {
    const int rows_on = STEP / cols, cols_on = STEP % cols;
    int r = first / cols, c = first % cols;
#pragma unroll 8
    while (r < rows) {
      if (!skip(r)) take(x[r * ld + c]);
      r += rows_on, c += cols_on;
      if (c >= cols) c -= cols, ++r;
    }
  }
  return group_max(m, lds);
}

// First kernel of a backward pass: the largest finite |dloss| of the rows that count (a row whose dloss is NaN or
// infinite keeps it in its dl / ref), and for fp32 the ranges of the classes of W
// and of the rows of h that count, or a copy of h in which the other rows are zeros.
__global__ __launch_bounds__(1024) void k_loss_range(const float* __restrict__ w, long w_ld,
                                                     const float* __restrict__ bias, const float* __restrict__ h,
                                                     long h_ld, int features, Rows g,
                                                     const float* __restrict__ dloss, Numbers* __restrict__ to,
                                                     float* __restrict__ copy) {
  __shared__ float lds[16];
  if (copy) {
    for (int r = blockIdx.x; r < g.rows; r += gridDim.x) {
      const bool kept = g.kept(r);
      for (int c = threadIdx.x; c < features; c += 1024)
        copy[(long)r * features + c] = kept ? h[(long)r * h_ld + c] : 0.f;
    }
    h = nullptr;
  }
  if (dloss && blockIdx.x == 0) {
    float m = 0;
    for (int t = threadIdx.x; t < g.rows; t += 1024)
      if (const float v = __builtin_fabsf(dloss[t]); v < kInf && g.kept(t)) m = __builtin_fmaxf(m, v);
    m = group_max(m, lds);
    if (threadIdx.x == 0) to->ref = m > 0 ? m : 1.f;
  }
  if (w) {
    // A class that a bias of -infinity masks has a gradient only where it is a target.
    float m = 0;
    if (bias)
      for (int t = blockIdx.x * 1024 + threadIdx.x; t < g.rows; t += kRange * 1024)
        if (g.kept(t) && masked(bias, (int)g.target[t]))
          for (int c = 0; c < features; ++c) {
            const float v = __builtin_fabsf(w[g.target[t] * w_ld + c]);
            m = v < kInf ? __builtin_fmaxf(m, v) : m;
          }
    m = range_of(w, w_ld, g.classes, features, !bias, [&](int v) { return masked(bias, v); }, m, lds);
    if (threadIdx.x == 0) to->max_w[blockIdx.x] = m;
  }
  if (h) {
    const float m = range_of(h, h_ld, g.rows, features, false, [&](int t) { return !g.kept(t); }, 0.f, lds);
    if (threadIdx.x == 0) to->max_h[blockIdx.x] = m;
  }
}

// One tensor to planes: [rows][cols] -> rows of ld elements, columns from cols to ld zero.
struct Copy {
  const void* src;
  long src_ld;
  int rows, cols;
  uint16_t* dst;
  int ld;
  int masked;             // rows of h that do not count as zeros
  const float* most;      // fp32: [kRange] partial maxima; null: one power of two a row
  int* exponent;          // the one or the rows'
};

// x in a plane's units.  Finite values beyond the range, which only classes without a gradient hold, stay finite:
// zeros multiply them.
__device__ __forceinline__ float within(float x, float scale) {
  const float v = x * scale;
  return __builtin_fabsf(x) < kInf ? __builtin_fminf(__builtin_fmaxf(v, -32768.f), 32768.f) : v;
}

template <class T, int NP>
__device__ __forceinline__ void copy_rows(const Copy& o, const Rows& g, unsigned block, unsigned blocks, float* lds) {
  float scale = 1;
  if constexpr (NP == 2) {
    const int e = exponent_for(group_max(o.most[threadIdx.x], lds));
    scale = power(e);
    if (block == 0 && threadIdx.x == 0) *o.exponent = e;
  }
  const unsigned each = o.ld / 8;
  const long items = (long)o.rows * each;
  for (long i = (long)block * 256 + threadIdx.x; i < items; i += (long)blocks * 256) {
    const long r = i >> 32 ? i / each : (long)((unsigned)i / each);
    const int c = (int)(i - r * each) * 8;
    const bool in = !o.masked || g.kept((int)r);
    __attribute__((aligned(16))) uint16_t out[NP][8];
    const T* p = static_cast<const T*>(o.src) + r * o.src_ld + c;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t q[NP] = {};
      if (in && c + e < o.cols) {
        if constexpr (NP == 1) q[0] = p[e];
        else cut<2>(within(p[e], scale), q);
      }
#pragma unroll
      for (int n = 0; n < NP; ++n) out[n][e] = q[n];
    }
#pragma unroll
    for (int n = 0; n < NP; ++n)
      *reinterpret_cast<uint4*>(o.dst + r * o.ld * NP + place<NP>(c) + n * 32) = *reinterpret_cast<const uint4*>(out[n]);
  }
}

// fp32 rows, each under a power of two of its own: one wave a row.
__device__ __forceinline__ void copy_rows_apart(const Copy& o, unsigned block, unsigned blocks) {
  const int lane = threadIdx.x & 63;
  for (long r = (long)block * 4 + (threadIdx.x >> 6); r < o.rows; r += (long)blocks * 4) {
    const float* p = static_cast<const float*>(o.src) + r * o.src_ld;
    float m = 0;
#pragma unroll 8
    for (int c = lane; c < o.cols; c += 64) {
      const float v = __builtin_fabsf(p[c]);
      m = v < kInf ? __builtin_fmaxf(m, v) : m;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, d, 64));
    const int e = exponent_for(m);
    const float scale = power(e);
    if (lane == 0) o.exponent[r] = e;
#pragma unroll 4
    for (int c = lane * 2; c < o.ld; c += 128) {
      uint16_t a[2], b[2];
      cut<2>(c < o.cols ? p[c] * scale : 0.f, a);
      cut<2>(c + 1 < o.cols ? p[c + 1] * scale : 0.f, b);
#pragma unroll
      for (int n = 0; n < 2; ++n)
        *reinterpret_cast<ushort2*>(o.dst + r * o.ld * 2 + place<2>(c) + n * 32) = make_ushort2(a[n], b[n]);
    }
  }
}

// W's piece and h to planes in one launch: the first `first` work groups take W.
template <class T, int NP>
__global__ __launch_bounds__(256) void k_loss_planes(Copy w, Copy h, unsigned first, Rows g) {
  __shared__ float lds[4];
  const bool of_w = blockIdx.x < first;
  const Copy o = of_w ? w : h;
  const unsigned block = of_w ? blockIdx.x : blockIdx.x - first, blocks = of_w ? first : gridDim.x - first;
  if (NP == 2 && !o.most) copy_rows_apart(o, block, blocks);
  else copy_rows<T, NP>(o, g, block, blocks, lds);
}

// What the logits of a piece need besides the operands.
struct Logits {
  const float* bias;         // of all classes, may be null
  Rows g;
  int first, count;          // classes of this piece
  int k;                     // features in whole stages
  const int* of_w;           // fp32: the planes' exponents, one for all rows or (apart) one a row
  const int* of_h;
  int apart;
};

// Products -> logits of a tile: units, bias, and -infinity beyond the last class.
template <class T>
__device__ __forceinline__ void to_logits(const Logits& g, int v0, int j_t, f32x4 (&acc)[T::TM][T::TN], int j) {
  if constexpr (T::NP == 2) {
    const int u = g.of_h[g.apart ? j_t : 0];
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = v0 + i * 16 + e;
        acc[i][j][e] = __builtin_ldexpf(acc[i][j][e], -(u + g.of_w[!g.apart ? 0 : v < g.count ? v : g.count - 1]));
      }
  }
  if (g.bias || v0 + T::TM * 16 > g.count) {
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = v0 + i * 16 + e;
        if (v >= g.count) {
          acc[i][j][e] = -kInf;
        } else if (g.bias) {
          const float b = g.bias[g.first + v];
          acc[i][j][e] = b == -kInf ? b : acc[i][j][e] + b;   // also where the product overflows
        }
      }
  }
}

// A row's lse from its maximum and its sum of exponentials, and its loss from that and its target's logit.
__device__ __forceinline__ void finish_row(const Rows& g, int t, float top, float sum, const float* hit, float* loss,
                                           float* lse) {
  const float all = (top == -kInf ? 0.f : top) + __builtin_logf(sum);   // log 0 = -inf: every class masked
  lse[t] = all;
  float v = 0;
  if (g.kept(t)) v = hit[t] == -kInf && !(all != all) ? kInf : all - hit[t];
  loss[t] = v;
}

// Forward: best[part][t], part = tile of classes: maximum and sum of exp(l - maximum); the target's
// logit of every row that has one.  With one tile of classes in all (loss given) the rows are finished
// here.
template <class T>
__global__ __launch_bounds__(T::THREADS) void k_loss_logits(Operand w, Operand h, Logits g, int tiles_m,
                                                            int tiles_n, int part0, float2* __restrict__ best,
                                                            float* hit, float* __restrict__ loss,
                                                            float* __restrict__ lse) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  int tm, tn;
  tile_at(place_of_group(blockIdx.x, tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(w, h, 0, m0, n0, 0, g.k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
  __syncthreads();
  float2* join = reinterpret_cast<float2*>(lds);   // [WM][BN]
  const int v0 = m0 + wm * T::TM * 16 + (lane >> 4) * 4;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int t = n0 + (wn * T::TN + j) * 16 + (lane & 15);
    const int row = t < g.g.rows ? t : g.g.rows - 1;
    to_logits<T>(g, v0, row, acc, j);
    // the target, counted from this lane's first class
    const long off = t < g.g.rows && g.g.kept(t) ? g.g.target[t] - g.first - v0 : -1;
    if (__any(off >= 0 && off < T::TM * 16)) {
#pragma unroll
      for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (off == i * 16 + e) hit[t] = acc[i][j][e];
    }
    float top = -kInf;
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = __builtin_fmaxf(top, acc[i][j][e]);
#pragma unroll
    for (int d = 16; d < 64; d *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, d, 64));
    const float base = top == -kInf ? 0.f : top;
    float sum = 0;
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += exp_of(acc[i][j][e] - base);
#pragma unroll
    for (int d = 16; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    if (lane < 16) join[wm * T::BN + (wn * T::TN + j) * 16 + lane] = make_float2(top, sum);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < T::BN; i += T::THREADS) {
    float top = join[i].x, sum = 0;
#pragma unroll
    for (int q = 1; q < T::WM; ++q) top = __builtin_fmaxf(top, join[q * T::BN + i].x);
    const float base = top == -kInf ? 0.f : top;
#pragma unroll
    for (int q = 0; q < T::WM; ++q) sum += join[q * T::BN + i].y * exp_of(join[q * T::BN + i].x - base);
    if (n0 + i >= g.g.rows) continue;
    if (loss) finish_row(g.g, n0 + i, top, sum, hit, loss, lse);   // hit: written before the barrier
    else best[(long)(part0 + tm) * g.g.rows + n0 + i] = make_float2(top, sum);
  }
}

// The parts of a row -> loss and lse.  256 / EACH rows a work group, EACH threads a row.
template <int EACH>
__global__ __launch_bounds__(256) void k_loss_join(const float2* __restrict__ best, int parts,
                                                   const float* __restrict__ hit, Rows g, float* __restrict__ loss,
                                                   float* __restrict__ lse) {
  constexpr int ROWS = 256 / EACH;
  __shared__ float lds[2][EACH][ROWS];
  const int x = threadIdx.x % ROWS, y = threadIdx.x / ROWS;
  const int t = blockIdx.x * ROWS + x;
  float top = -kInf, sum = 0;
  if (t < g.rows)
    for (int p = y; p < parts; p += EACH) top = __builtin_fmaxf(top, best[(long)p * g.rows + t].x);
  lds[0][y][x] = top;
  __syncthreads();
  for (int d = EACH / 2; d > 0; d /= 2) {
    if (y < d) lds[0][y][x] = __builtin_fmaxf(lds[0][y][x], lds[0][y + d][x]);
    __syncthreads();
  }
  top = lds[0][0][x];
  const float base = top == -kInf ? 0.f : top;
  if (t < g.rows)
    for (int p = y; p < parts; p += EACH) {
      const float2 b = best[(long)p * g.rows + t];
      sum += b.y * exp_of(b.x - base);
    }
  lds[1][y][x] = sum;
  __syncthreads();
  for (int d = EACH / 2; d > 0; d /= 2) {
    if (y < d) lds[1][y][x] += lds[1][y + d][x];
    __syncthreads();
  }
  if (y != 0 || t >= g.rows) return;
  finish_row(g, t, top, lds[1][0][x], hit, loss, lse);
}

// Backward: dl / ref of a piece, rows [t][ld]; `rest`, may be null: what bf16 leaves of it; the sums over a
// wave's rows for dbias.
template <class T>
__global__ __launch_bounds__(T::THREADS) void k_loss_dlogits(Operand w, Operand h, Logits g, int tiles_m,
                                                             int tiles_n, const float* __restrict__ lse,
                                                             const float* __restrict__ dloss,
                                                             const float* __restrict__ ref,
                                                             uint16_t* __restrict__ dl, int ld,
                                                             uint16_t* __restrict__ rest,
                                                             float* __restrict__ dbias) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  int tm, tn;
  tile_at(place_of_group(blockIdx.x, tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(w, h, 0, m0, n0, 0, g.k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
  const float scale = *ref;
  const int v0 = m0 + wm * T::TM * 16 + (lane >> 4) * 4;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int t = n0 + (wn * T::TN + j) * 16 + (lane & 15);
    const int row = t < g.g.rows ? t : g.g.rows - 1;
    to_logits<T>(g, v0, row, acc, j);
    const bool kept = t < g.g.rows && g.g.kept(row);
    const float all = kept ? lse[row] : 0.f;
    const float weight = kept && all != -kInf ? dloss[row] / scale : 0.f;
    const long off = kept ? g.g.target[row] - g.first - v0 : -1;
    const bool near = __any(off >= 0 && off < T::TM * 16);
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      f32x4 d = acc[i][j];
#pragma unroll
      for (int e = 0; e < 4; ++e) d[e] = exp_of(d[e] - all);
      if (near)
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] -= off == i * 16 + e ? 1.f : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) d[e] = weight == 0.f ? 0.f : d[e] * weight;   // of a row that is left out: zeros
      acc[i][j] = d;
      const int v = v0 + i * 16;
      if (t >= g.g.rows || v >= ld) continue;   // ld is a multiple of 4; from the last class on d is zero
      // tiles of 32 end where the line's last ones have no rows of W: zeros behind them
      const bool pad = is_few<T> && tm + 1 == tiles_m && v + 32 < ld;
      if constexpr (T::NP == 3) {
        float* to = reinterpret_cast<float*>(dl) + (long)t * ld + v;
        *reinterpret_cast<f32x4*>(to) = d;
        if (pad) *reinterpret_cast<f32x4*>(to + 32) = f32x4{0, 0, 0, 0};
      } else {
        uint16_t out[4][T::NP];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (T::NP == 2) cut<2>(d[e] * (float)(1 << kDlExponent), out[e]);
          else cut<1>(d[e], out[e]);
        }
#pragma unroll
        for (int p = 0; p < T::NP; ++p)
          *reinterpret_cast<ushort4*>(dl + (long)t * ld * T::NP + place<T::NP>(v) + p * 32) =
              make_ushort4(out[0][p], out[1][p], out[2][p], out[3][p]);
        if (T::NP == 1 && rest)
          *reinterpret_cast<ushort4*>(rest + (long)t * ld + v) =
              make_ushort4(bf16_bits(d[0] - bf16_value(out[0][0])), bf16_bits(d[1] - bf16_value(out[1][0])),
                           bf16_bits(d[2] - bf16_value(out[2][0])), bf16_bits(d[3] - bf16_value(out[3][0])));
        if (pad) {
#pragma unroll
          for (int p = 0; p < T::NP; ++p)
            *reinterpret_cast<ushort4*>(dl + (long)t * ld * T::NP + place<T::NP>(v + 32) + p * 32) = make_ushort4(0, 0, 0, 0);
          if (T::NP == 1 && rest) *reinterpret_cast<ushort4*>(rest + (long)t * ld + v + 32) = make_ushort4(0, 0, 0, 0);
        }
      }
    }
  }
  if (!dbias) return;
#pragma unroll
  for (int i = 0; i < T::TM; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float s = acc[i][0][e];
#pragma unroll
      for (int j = 1; j < T::TN; ++j) s += acc[i][j][e];
#pragma unroll
      for (int d = 1; d < 16; d *= 2) s += __shfl_xor(s, d, 64);
      const int v = v0 + i * 16 + e;
      if ((lane & 15) == 0 && v < g.count) dbias[(long)(tn * T::WN + wn) * g.g.classes + g.first + v] = s;
    }
}

// The gradient of the rows of h or W: out[row][f] = sum_k A(row, k) B(f, k) over the features f.
// kind 0: to fp32, 1: to bf16, both times ref; 2: to fp32 sums of a range of k (blockIdx.y), kept as
// they are, 3: added to what is there.  A lane of the instruction's result holds four consecutive m of
// one n.  FOUR: m are the features, four of them one store (rows of out start on whole fours); otherwise
// m are the rows, and sixteen lanes store neighbouring features.  (dW of 2048 x 1024 x 16384 in bf16: 71 us and 78,
// of a piece of 4096 x 2048 x 32768 574 and 580, of 4096 x 2048 x 8192 in fp32 326 and 329; dh there 84 and 84, 538 and
// 531, 349 and 349; dW of 10007 x 515 in fp32, whose rows start anywhere: 60 and 55.)
struct Product {
  Operand rows, features;
  const uint16_t* rest;  // of `rows`, may be null: a second product on top of the first
  void* out;
  long split;            // elements between ranges of k
  int kind, k, per;      // k in all and per range
  int count, width;      // rows and features of out
  const float* ref;
  const int* exponent;   // of the features' planes
};
template <class T, bool FOUR>
__device__ __forceinline__ void make_product(const Product& p, int group, int groups, int range, char* lds) {
  const Operand& a = FOUR ? p.features : p.rows;
  const Operand& b = FOUR ? p.rows : p.features;
  const int all_m = FOUR ? p.width : p.count, all_n = FOUR ? p.count : p.width;
  int tm, tn;
  tile_at(place_of_group(group, groups), (all_m + T::BM - 1) / T::BM, (all_n + T::BN - 1) / T::BN, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  const int k0 = range * p.per, k1 = k0 + p.per < p.k ? k0 + p.per : p.k;
  if (T::NP == 1 && p.rest) {   // the smaller one first
    Operand rest = p.rows;
    rest.p = p.rest;
    multiply<T>(FOUR ? a : rest, FOUR ? rest : b, 0, m0, n0, k0, k1, lds, acc);
    __syncthreads();
  }
  multiply<T>(a, b, 0, m0, n0, k0, k1, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
  const float scale = p.kind < 2 ? *p.ref : 1.f;
  const int e2 = T::NP == 2 ? -(*p.exponent + kDlExponent) : 0;
  const long base = range * p.split;
#pragma unroll
  for (int i = 0; i < T::TM; ++i) {
    const int m = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4;
    if (m >= all_m) continue;
#pragma unroll
    for (int j = 0; j < T::TN; ++j) {
      const int n = n0 + (wn * T::TN + j) * 16 + (lane & 15);
      if (n >= all_n) continue;
      f32x4 v = acc[i][j];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (T::NP == 2 ? __builtin_ldexpf(v[e], e2) : v[e]) * scale;
      if constexpr (FOUR) {
        const long at = base + (long)n * p.width + m;
        if (p.kind == 1) {
          *reinterpret_cast<ushort4*>(static_cast<uint16_t*>(p.out) + at) =
              make_ushort4(bf16_bits(v[0]), bf16_bits(v[1]), bf16_bits(v[2]), bf16_bits(v[3]));
        } else {
          f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at);
          if (p.kind == 3) v += *o;
          *o = v;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (m + e >= all_m) continue;
          const long at = base + (long)(m + e) * p.width + n;
          if (p.kind == 1) static_cast<uint16_t*>(p.out)[at] = bf16_bits(v[e]);
          else if (p.kind == 3) static_cast<float*>(p.out)[at] += v[e];
          else static_cast<float*>(p.out)[at] = v[e];
        }
      }
    }
  }
}
template <class T, bool FOUR>
__global__ __launch_bounds__(T::THREADS) void k_loss_product(Product p) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  make_product<T, FOUR>(p, blockIdx.x, gridDim.x, blockIdx.y, lds);
}
// dh and dW of a piece in one launch, where both have few tiles and would each leave compute units idle
// (2048 x 64 x 1000 in fp32, a training step: 63 us, with two launches 70; 59 x 4081 x 25462: 582 and 609): the first `first` work groups have dh's
// tiles and ranges, the others dW's.
template <class H, class W>
__global__ __launch_bounds__(H::THREADS) void k_loss_products(Product h, Product w, int first, int tiles_h,
                                                              int tiles_w) {
  static_assert(H::THREADS == W::THREADS);
  __shared__ __attribute__((aligned(1024))) char lds[H::LDS > W::LDS ? H::LDS : W::LDS];
  const int b = blockIdx.x;
  if (b < first) make_product<H, false>(h, b % tiles_h, tiles_h, b / tiles_h, lds);
  else make_product<W, false>(w, (b - first) % tiles_w, tiles_w, (b - first) / tiles_w, lds);
}

// Sums of the ranges of k -> dh or dW (the first `first` work groups), and, as the backward pass's last kernel,
// of the waves' rows -> dbias.
__global__ __launch_bounds__(256) void k_loss_sums(const float* __restrict__ sums, int count, long items, int bf16,
                                                   void* __restrict__ out, unsigned first,
                                                   const float* __restrict__ parts, int part_count, int classes,
                                                   float* __restrict__ dbias, const float* __restrict__ ref) {
  const float scale = *ref;
  if (blockIdx.x < first) {
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long)first * 256) {
      float s = 0;
#pragma unroll 8
      for (int q = 0; q < count; ++q) s += sums[q * items + i];
      s *= scale;
      if (bf16) static_cast<uint16_t*>(out)[i] = bf16_bits(s);
      else static_cast<float*>(out)[i] = s;
    }
  } else {
    const long step = (long)(gridDim.x - first) * 256;
    for (long v = (long)(blockIdx.x - first) * 256 + threadIdx.x; v < classes; v += step) {
      float s = 0;
#pragma unroll 4
      for (int p = 0; p < part_count; ++p) s += parts[(long)p * classes + v];
      dbias[v] = s * scale;
    }
  }
}

__global__ __launch_bounds__(256) void k_loss_zero(uint16_t* p, long items) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long)gridDim.x * 256) p[i] = 0;
}

unsigned grid_of(long items, long most) {
  const long b = (items + 255) / 256;
  return (unsigned)(b < 1 ? 1 : b < most ? b : most);
}

// Tiles.  256 x 256 where they fill the chip, else 128 x 128, else 64 x 64 (and two to five work
// groups a compute unit).
template <int NP, bool AX, bool BX>
struct Tiles {
  typedef Tile<256, 256, 2, 4, NP, 2, AX, BX> Big;
  typedef Tile<128, 128, 2, 2, NP, 2, AX, BX> Mid;
  typedef Tile<64, 64, 2, 2, NP, 2, AX, BX> Small;
  typedef Tile<64, 64, 2, 2, NP, 4, AX, BX> Deep;   // where two work groups a compute unit are all there are
};
// (A training step of 900 x 4092 x 401 in bf16: 104 us, all of ring 2 125; of 3 x 925 x 75113 in fp32: 328, all of
// ring 4 428.)
constexpr long kDeepGroups = 512;

template <int NP, bool AX, bool BX, class F>
void with_tile(int side, long groups, F&& f) {
  if constexpr (NP < 3) {
    if (side == 256) return f(typename Tiles<NP, AX, BX>::Big{});
    if (side == 128) return f(typename Tiles<NP, AX, BX>::Mid{});
  }
  if constexpr (!AX && !BX)
    if (side == 32) return f(Few<NP>{});
  if (groups <= kDeepGroups) f(typename Tiles<NP, AX, BX>::Deep{});
  else f(typename Tiles<NP, AX, BX>::Small{});
}

// bf16 rows that the products can take where they lie: 16-byte accesses, whole stages of k.
bool direct(const LossArgs& a, const void* p, long stride) {
  return a.bf16 && a.features % 64 == 0 && stride % 8 == 0 && stride <= kMaxLd && ((uintptr_t)p & 15) == 0;
}

const void* row_at(const LossArgs& a, const void* p, long row, long stride) {
  return static_cast<const char*>(p) + row * stride * (a.bf16 ? 2 : 4);
}

// What k of the logits runs to: rows of planes are padded to whole lines of 64 or two of 32, tensors that are
// read as they stand are not, and no stage may lie behind their rows.
template <int NP>
int logits_k(const LossArgs& a, const LossLayout& l) { return NP == 3 ? whole_stages_of_32(a.features) : l.dp; }

// Operands of a piece: where they lie, or planes made here.
template <int NP>
void operands(const LossArgs& a, const LossLayout& l, const Rows& g, const void* w_rows, int count, const void* h,
              bool w_direct, bool h_ready, bool back, Numbers* num, char* ws, Operand* ow, Operand* oh,
              hipStream_t st) {
  if constexpr (NP == 3) {
    *ow = Operand{(const uint16_t*)w_rows, a.w_stride * 2, 0, count, a.features};
    *oh = back ? Operand{(const uint16_t*)(ws + l.h), a.features * 2L, 0, a.rows, a.features}
               : Operand{(const uint16_t*)h, a.h_stride * 2, 0, a.rows, a.features};
  } else {
  uint16_t* to_w = reinterpret_cast<uint16_t*>(ws + l.w);
  uint16_t* to_h = reinterpret_cast<uint16_t*>(ws + l.h);
  const long pw = (long)count * l.dp / 8, ph = (long)a.rows * l.dp / 8;
  const Copy cw{w_rows, a.w_stride, count, a.features, to_w, l.dp, 0, back ? num->max_w : nullptr,
                back ? &num->of_w : reinterpret_cast<int*>(ws + l.unit_w)};
  const Copy ch{h, a.h_stride, a.rows, a.features, to_h, l.dp, back, back ? num->max_h : nullptr,
                back ? &num->of_h : reinterpret_cast<int*>(ws + l.unit_h)};
  // a wave a row, or a thread eight values
  const auto grid = [&](long rows, long eights) { return NP == 2 && !back ? grid_of(rows * 64, 2048) : grid_of(eights, 2048); };
  const unsigned first = w_direct ? 0 : grid(count, pw), more = h_ready ? 0 : grid(a.rows, ph);
  typedef typename std::conditional<NP == 1, uint16_t, float>::type T;
  if (first + more) wino_launch((k_loss_planes<T, NP>), dim3(first + more), dim3(256), st, cw, ch, first, g);
  *ow = w_direct ? Operand{(const uint16_t*)w_rows, a.w_stride, 0, count, a.features}
                 : Operand{to_w, (long)l.dp * NP, 0, count, l.dp};
  if (!h_ready) *oh = Operand{to_h, (long)l.dp * NP, 0, a.rows, l.dp};
  }
}

template <int NP>
hipError_t forward(const LossArgs& a, const void* h, const void* w, const float* bias, const int64_t* target,
                   float* loss, float* lse, char* ws, hipStream_t st) {
  const LossLayout l = loss_layout(a, false);
  Numbers* num = reinterpret_cast<Numbers*>(ws + l.numbers);
  float2* best = reinterpret_cast<float2*>(ws + l.parts);
  float* hit = reinterpret_cast<float*>(ws + l.target);
  const Rows g{target, a.ignore_index, a.rows, a.classes};
  const bool w_direct = direct(a, w, a.w_stride);
  bool h_ready = direct(a, h, a.h_stride);
  Operand oh{(const uint16_t*)h, a.h_stride, 0, a.rows, a.features}, ow{};
  // a launch holds fewer than 2^32 threads
  const long most = (1L << 21) / ((a.rows + 63) / 64) * 64;
  long piece = w_direct || NP == 3 ? a.classes : l.piece;
  if (piece > most) piece = most < 256 ? 256 : most / 256 * 256;
  Logits q{bias, g, 0, 0, logits_k<NP>(a, l), reinterpret_cast<const int*>(ws + l.unit_w), reinterpret_cast<const int*>(ws + l.unit_h), 1};
  int part = 0;
  for (long first = 0; first < a.classes; first += piece) {
    q.first = (int)first;
    q.count = (int)(a.classes - first < piece ? a.classes - first : piece);
    operands<NP>(a, l, g, row_at(a, w, first, a.w_stride), q.count, h, w_direct, h_ready, false, num, ws, &ow, &oh, st);
    h_ready = true;
    with_tile<NP, false, false>(logits_side(a, l, q.count),
                                count_of(q.count, a.rows, 64), [&](auto tile) {
      typedef decltype(tile) T;
      const int tm = (q.count + T::BM - 1) / T::BM, tn = (a.rows + T::BN - 1) / T::BN;
      const bool all = tm == 1 && q.count == a.classes;
      wino_launch((k_loss_logits<T>), dim3(tm * tn), dim3(T::THREADS), st, ow, oh, q, tm, tn, part, best, hit,
                  all ? loss : nullptr, lse);
      part += all ? 0 : tm;
    });
  }
  if (part == 0) return hipGetLastError();
  // few rows: all threads of a work group on one
  if (a.rows >= 1024)
    wino_launch((k_loss_join<16>), dim3((a.rows + 15) / 16), dim3(256), st, (const float2*)best, part, (const float*)hit,
                g, loss, lse);
  else
    wino_launch((k_loss_join<256>), dim3(a.rows), dim3(256), st, (const float2*)best, part, (const float*)hit, g, loss,
                lse);
  return hipGetLastError();
}

template <int NP>
hipError_t backward(const LossArgs& a, const void* h, const void* w, const float* bias, const int64_t* target,
                    const float* lse, const float* dloss, void* dh, void* dw, float* dbias, char* ws,
                    hipStream_t st) {
  const LossLayout l = loss_layout(a, true);
  Numbers* num = reinterpret_cast<Numbers*>(ws + l.numbers);
  const float* ref = &num->ref;
  const Rows g{target, a.ignore_index, a.rows, a.classes};
  wino_launch(k_loss_range, dim3(NP == 1 ? 1 : kRange), dim3(1024), st, NP == 2 ? (const float*)w : nullptr, a.w_stride,
              bias, NP == 1 ? nullptr : (const float*)h, a.h_stride, a.features, g, dloss, num,
              NP == 3 ? reinterpret_cast<float*>(ws + l.h) : nullptr);
  const bool w_direct = direct(a, w, a.w_stride);
  bool h_ready = false;   // always a copy: rows that are left out as zeros
  Operand oh{}, ow{};
  Logits q{bias, g, 0, 0, logits_k<NP>(a, l), &num->of_w, &num->of_h, 0};
  uint16_t* dl = reinterpret_cast<uint16_t*>(ws + l.dl);
  uint16_t* rest = l.two ? reinterpret_cast<uint16_t*>(ws + l.rest) : nullptr;
  float* db = dbias ? reinterpret_cast<float*>(ws + l.dbias) : nullptr;
  float* sums = reinterpret_cast<float*>(ws + l.dh);
  const bool one = l.splits == 1 && l.piece >= a.classes;   // dh comes from one product
  int parts = 0;
  for (long first = 0; first < a.classes; first += l.piece) {
    q.first = (int)first;
    q.count = a.classes - q.first < l.piece ? a.classes - q.first : l.piece;
    const int vp = (int)up(q.count, 64);
    operands<NP>(a, l, g, row_at(a, w, first, a.w_stride), q.count, h, w_direct, h_ready, true, num, ws, &ow, &oh, st);
    h_ready = true;
    with_tile<NP, false, false>(l.side, count_of(q.count, a.rows, 64), [&](auto tile) {
      typedef decltype(tile) T;
      const int tm = (q.count + T::BM - 1) / T::BM, tn = (a.rows + T::BN - 1) / T::BN;
      parts = tn * T::WN;
      wino_launch((k_loss_dlogits<T>), dim3(tm * tn), dim3(T::THREADS), st, ow, oh, q, tm, tn, lse, dloss, ref, dl, vp,
                  rest, db);
    });
    const Operand od{dl, (long)vp * (NP == 1 ? 1 : 2), 0, a.rows, vp};
    const int per = (int)up((vp + l.splits - 1) / l.splits, 64), tk = (int)up(a.rows, 64);
    const int dw_per = (int)up((tk + l.dw_splits - 1) / l.dw_splits, 64);
    float* dw_sums = l.dw_splits > 1 ? reinterpret_cast<float*>(ws + l.dw) : nullptr;
    void* dw_rows = dw ? const_cast<void*>(row_at(a, dw, first, a.features)) : nullptr;
    const long dw_items = (long)q.count * a.features;
    const Product ph{od, ow, rest, one ? dh : (void*)sums, (long)a.rows * a.features, one ? a.bf16 : first ? 3 : 2, vp, per,
                     a.rows, a.features, ref, &num->of_w};
    const Product pw{od, oh, rest, dw_sums ? (void*)dw_sums : dw_rows, dw_items, dw_sums ? 2 : a.bf16, tk, dw_per, q.count,
                     a.features, ref, &num->of_h};
    const int side_w = dw_side(a, l, q.count);
    const auto tiles = [](const Product& p, int side) { return (int)count_of(p.count, p.width, side); };
    if (dh && dw && l.dh_side == 64 && side_w == 64) {
      const int th = tiles(ph, 64), tw = tiles(pw, 64), all = th * l.splits;
      const auto launch = [&](auto h, auto w) {
        typedef decltype(h) H;
        typedef decltype(w) W;
        wino_launch((k_loss_products<H, W>), dim3(all + tw * l.dw_splits), dim3(H::THREADS), st, ph, pw, all, th, tw);
      };
      if (all + tw * l.dw_splits <= kDeepGroups)
        launch(typename Tiles<NP, false, true>::Deep{}, typename Tiles<NP, true, true>::Deep{});
      else
        launch(typename Tiles<NP, false, true>::Small{}, typename Tiles<NP, true, true>::Small{});
    } else {
      // tiles of 64 as in the launch of both, so that a gradient's bits do not go by which others are asked for
      const auto whole = [&](const Product& p, int side) {
        return side > 64 && a.features % 4 == 0 && ((uintptr_t)p.out & (p.kind == 1 ? 7 : 15)) == 0;
      };
      const auto launch = [&](auto tile, auto four, const Product& p, int ranges) {
        typedef decltype(tile) T;
        wino_launch((k_loss_product<T, decltype(four)::value>), dim3(tiles(p, T::BM), ranges), dim3(T::THREADS), st, p);
      };
      const long groups_h = (long)tiles(ph, 64) * l.splits, groups_w = (long)tiles(pw, 64) * l.dw_splits;
      if (dh && whole(ph, l.dh_side))
        with_tile<NP, true, false>(l.dh_side, groups_h, [&](auto t) { launch(t, std::true_type{}, ph, l.splits); });
      else if (dh)
        with_tile<NP, false, true>(l.dh_side, groups_h, [&](auto t) { launch(t, std::false_type{}, ph, l.splits); });
      if (dw)
        with_tile<NP, true, true>(side_w, groups_w, [&](auto t) {
          if (whole(pw, side_w)) launch(t, std::true_type{}, pw, l.dw_splits);
          else launch(t, std::false_type{}, pw, l.dw_splits);
        });
    }
    if (dw && dw_sums) {
      const unsigned grid = grid_of(dw_items, 8192);
      wino_launch(k_loss_sums, dim3(grid), dim3(256), st, (const float*)dw_sums, l.dw_splits, dw_items, a.bf16, dw_rows, grid,
                  (const float*)nullptr, 0, 0, (float*)nullptr, ref);
    }
  }
  const long items = (long)a.rows * a.features;
  const unsigned first = dh && !one ? grid_of(items, 8192) : 0, more = dbias ? grid_of(a.classes, 1024) : 0;
  if (first + more)
    wino_launch(k_loss_sums, dim3(first + more), dim3(256), st, (const float*)sums, l.splits, items, a.bf16, dh, first,
                (const float*)db, parts, a.classes, dbias, ref);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_loss(const LossArgs& a, const void* h, const void* w, const float* bias,
                       const int64_t* target, float* loss, float* lse, char* ws, hipStream_t st) {
  return a.bf16 ? forward<1>(a, h, w, bias, target, loss, lse, ws, st)
       : as_it_stands(a) ? forward<3>(a, h, w, bias, target, loss, lse, ws, st)
                         : forward<2>(a, h, w, bias, target, loss, lse, ws, st);
}

hipError_t launch_loss_backward(const LossArgs& a, const void* h, const void* w, const float* bias,
                                const int64_t* target, const float* lse, const float* dloss, void* dh,
                                void* dw, float* dbias, char* ws, hipStream_t st) {
  if (a.rows == 0) {   // no rows: the weights' gradient is zero
    const long items = (long)a.classes * a.features * (a.bf16 ? 1 : 2);
    if (dw) wino_launch(k_loss_zero, dim3(grid_of(items, 16384)), dim3(256), st, (uint16_t*)dw, items);
    if (dbias)
      wino_launch(k_loss_zero, dim3(grid_of(2L * a.classes, 16384)), dim3(256), st, (uint16_t*)dbias, 2L * a.classes);
    return hipGetLastError();
  }
  return a.bf16 ? backward<1>(a, h, w, bias, target, lse, dloss, dh, dw, dbias, ws, st)
       : as_it_stands(a) ? backward<3>(a, h, w, bias, target, lse, dloss, dh, dw, dbias, ws, st)
                         : backward<2>(a, h, w, bias, target, lse, dloss, dh, dw, dbias, ws, st);
}

}  // namespace wino
