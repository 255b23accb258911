// Softmax cross entropy of a linear classifier, h W^T + bias, without keeping the logits.
//
//   l = h W^T + b,  lse_t = log sum_v exp(l_tv),  loss_t = lse_t - l_t[target_t]
//   dl_tv = (exp(l_tv - lse_t) - [v = target_t]) dloss_t,  dh = dl W,  dW = dl^T h,  db = sum_t dl
//
// Forward: the logits of a tile leave the matrix instructions in registers and end there as a maximum
// and a sum of exponentials a row; those of all tiles are joined by a second kernel.  Backward: the
// logits are computed again, piece by piece of the classes, and become dl in the workspace, once as
// rows and once as columns, which are the operands of the two products of the piece.
//
// dl is kept on as many bf16 planes as the operands have (wino_products.hpp): one for bf16 operands,
// a rounding of half a step like the one that h, W and the gradients have; three, nothing lost, for
// fp32.  It is kept relative to the largest |dloss|, by which the products' results are multiplied in
// fp32: with one weight for all rows, as for a mean, the -1 of a target's class stays free of a
// rounding that would be the same in every row.
#include "wino_products.hpp"
#include "wino_train.hpp"

namespace wino {
namespace {

using namespace prod;

// exp(x) for x <= 0 or so: exp2 of x log2(e), the part of the product that fp32 loses added back.
__device__ __forceinline__ float exp_of(float x) {
  x = x < -150.f ? -150.f : x;   // a NaN stays one; exp(-150) is 0 in fp32
  const float t = x * 1.44269504f;
  const float r = __builtin_fmaf(x, 1.44269504f, -t) + x * 1.925963033e-8f;
  return __builtin_amdgcn_exp2f(t) * __builtin_fmaf(r, 0.69314718f, 1.f);
}

// src [rows][cols] (fp32 or bf16) -> planes [rows][ld], columns from cols to ld zero.
template <class T, int NP>
__global__ __launch_bounds__(256) void k_planes(const T* __restrict__ src, long src_ld, int rows, int cols,
                                                uint16_t* __restrict__ dst, long ld, long plane) {
  const long each = ld / 8;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < rows * each; i += (long)gridDim.x * 256) {
    const long r = i / each;
    const int c = (int)(i - r * each) * 8;
    __attribute__((aligned(16))) uint16_t out[NP][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t q[NP] = {};
      if (c + e < cols) {
        if constexpr (sizeof(T) == 2) q[0] = src[r * src_ld + c + e];
        else cut<NP>(src[r * src_ld + c + e], q);
      }
#pragma unroll
      for (int p = 0; p < NP; ++p) out[p][e] = q[p];
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
      *reinterpret_cast<uint4*>(dst + p * plane + r * ld + c) = *reinterpret_cast<const uint4*>(out[p]);
  }
}

// src [rows][cols] -> planes [cols][ld], dst[c][r] = src[r][c]; zero for r from rows to ld.  With
// `target`, rows whose target is no class count as zeros whatever they hold.
template <class T, int NP>
__global__ __launch_bounds__(256) void k_planes_across(const T* __restrict__ src, long src_ld, int rows,
                                                       int cols, uint16_t* __restrict__ dst, long ld,
                                                       long plane, const int64_t* __restrict__ target,
                                                       long ignore, int classes) {
  __shared__ T tile[64][64 + 4 / sizeof(T)];
  const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = r0 + y + i * 4, c = c0 + x;
    bool in = r < rows && c < cols;
    if (target && in) {
      const long t = target[r];
      in = t != ignore && t >= 0 && t < classes;
    }
    tile[y + i * 4][x] = in ? src[(long)r * src_ld + c] : (T)0;
  }
  __syncthreads();
  const int c = threadIdx.x >> 2, rq = (threadIdx.x & 3) * 16;
  if (c0 + c >= cols) return;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r = rq + half * 8;
    if (r0 + r >= ld) return;
    __attribute__((aligned(16))) uint16_t out[NP][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint16_t q[NP] = {};
      if constexpr (sizeof(T) == 2) q[0] = tile[r + e][c];
      else cut<NP>(tile[r + e][c], q);
#pragma unroll
      for (int p = 0; p < NP; ++p) out[p][e] = q[p];
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
      *reinterpret_cast<uint4*>(dst + p * plane + (long)(c0 + c) * ld + r0 + r) =
          *reinterpret_cast<const uint4*>(out[p]);
  }
}

// What the logits of a piece need besides the operands.
struct Logits {
  const float* bias;        // of all classes, may be null
  const int64_t* target;
  long ignore;
  int rows, classes;        // all of them
  int first;                // first class of this piece
  int count;                // classes of this piece
  int k;                    // features rounded up
};

// Work group of the grid -> tile (m of W's rows, n of h's rows).  Consecutive work groups go round
// robin over the 8 XCDs: each XCD takes a run of tiles, in which bands of eight tiles of classes keep
// their rows of W in its L2 while the rows of h pass.
__device__ __forceinline__ void tile_of(int tiles_m, int tiles_n, int& m, int& n) {
  const int all = tiles_m * tiles_n;
  int b = blockIdx.x;
  const int per = all / 8;
  if (b < per * 8) b = (b & 7) * per + (b >> 3);
  const int band = b / (8 * tiles_n), rest = b - band * 8 * tiles_n;
  const int wide = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
  m = band * 8 + rest % wide;
  n = rest / wide;
}

// Forward: best[part][t], part = tile of classes: maximum and sum of exp(l - maximum); the target's
// logit of every row that has one.
template <class T>
__global__ __launch_bounds__(T::THREADS) void k_loss_logits(Operand w, Operand h, Logits g, int tiles_m,
                                                            int tiles_n, int part0, float2* __restrict__ best,
                                                            float* __restrict__ hit) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  int tm, tn;
  tile_of(tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(w, h, 0, m0, n0, 0, g.k, g.k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
  __syncthreads();
  float2* join = reinterpret_cast<float2*>(lds);   // [WM][BN]
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int t = n0 + (wn * T::TN + j) * 16 + (lane & 15);
    const long cls = t < g.rows ? g.target[t] : -1;
    const bool kept = t < g.rows && cls != g.ignore && cls >= 0 && cls < g.classes;
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4 + e;
        float l = acc[i][j][e];
        if (v < g.count) {
          if (g.bias) l += g.bias[g.first + v];
          if (kept && cls == g.first + v) hit[t] = l;
        } else {
          l = -__builtin_inff();
        }
        acc[i][j][e] = l;
        top = __builtin_fmaxf(top, l);
      }
#pragma unroll
    for (int d = 16; d < 64; d *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, d, 64));
    const float base = top == -__builtin_inff() ? 0.f : top;
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
    const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int q = 0; q < T::WM; ++q)
      sum += join[q * T::BN + i].y * exp_of(join[q * T::BN + i].x - base);
    if (n0 + i < g.rows) best[(long)(part0 + tm) * g.rows + n0 + i] = make_float2(top, sum);
  }
}

// The parts of a row -> loss and lse.  16 rows a work group, 16 threads each.
__global__ __launch_bounds__(256) void k_loss_join(const float2* __restrict__ best, int parts,
                                                   const float* __restrict__ hit, Logits g,
                                                   float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float2 lds[16][16];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const int t = blockIdx.x * 16 + x;
  float top = -__builtin_inff(), sum = 0;
  if (t < g.rows)
    for (int p = y; p < parts; p += 16) {
      const float2 b = best[(long)p * g.rows + t];
      const float up = __builtin_fmaxf(top, b.x), base = up == -__builtin_inff() ? 0.f : up;
      sum = sum * exp_of(top - base) + b.y * exp_of(b.x - base);
      top = up;
    }
  lds[y][x] = make_float2(top, sum);
  __syncthreads();
  if (y != 0 || t >= g.rows) return;
  for (int q = 1; q < 16; ++q) top = __builtin_fmaxf(top, lds[q][x].x);
  const float base = top == -__builtin_inff() ? 0.f : top;
  sum = 0;
  for (int q = 0; q < 16; ++q) sum += lds[q][x].y * exp_of(lds[q][x].x - base);
  const float all = base + __builtin_logf(sum);   // log 0 = -inf: every class masked
  lse[t] = all;
  const long cls = g.target[t];
  const bool kept = cls != g.ignore && cls >= 0 && cls < g.classes;
  float v = 0;
  if (kept) v = hit[t] == -__builtin_inff() && !(all != all) ? __builtin_inff() : all - hit[t];
  loss[t] = v;
}

// The largest |dloss| of the rows that count.
__global__ __launch_bounds__(1024) void k_loss_weight(const float* __restrict__ dloss, Logits g,
                                                      float* __restrict__ ref) {
  __shared__ float lds[16];
  float m = 0;
  for (int t = threadIdx.x; t < g.rows; t += 1024) {
    const long cls = g.target[t];
    if (cls != g.ignore && cls >= 0 && cls < g.classes) m = __builtin_fmaxf(m, __builtin_fabsf(dloss[t]));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, d, 64));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) m = __builtin_fmaxf(m, lds[w]);
    *ref = m;
  }
}

// Backward: dl / ref of a piece, as rows dl [t][piece] and as columns dlt [v][tp]; the sums over a
// tile's rows for dbias.
template <class T>
__global__ __launch_bounds__(T::THREADS) void k_loss_dlogits(Operand w, Operand h, Logits g, int tiles_m,
                                                             int tiles_n, const float* __restrict__ lse,
                                                             const float* __restrict__ dloss,
                                                             const float* __restrict__ ref,
                                                             uint16_t* __restrict__ dl, long dl_ld, long dl_plane,
                                                             uint16_t* __restrict__ dlt, long dlt_ld,
                                                             long dlt_plane, float* __restrict__ dbias) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  int tm, tn;
  tile_of(tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  multiply<T>(w, h, 0, m0, n0, 0, g.k, g.k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
  const float scale = *ref;
  float sums[T::TM][4] = {};
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int t = n0 + (wn * T::TN + j) * 16 + (lane & 15);
    const long cls = t < g.rows ? g.target[t] : -1;
    const bool kept = t < g.rows && cls != g.ignore && cls >= 0 && cls < g.classes;
    const float all = kept ? lse[t] : 0.f;
    float weight = kept && all != -__builtin_inff() ? dloss[t] / scale : 0.f;
    if (scale == 0.f) weight = 0.f;
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      const int v = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4;
      uint16_t out[4][T::NP];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float d = 0;
        if (v + e < g.count && weight != 0.f) {
          float l = acc[i][j][e];
          if (g.bias) l += g.bias[g.first + v + e];
          d = (exp_of(l - all) - (cls == g.first + v + e ? 1.f : 0.f)) * weight;
        }
        sums[i][e] += d;
        cut<T::NP>(d, out[e]);
      }
#pragma unroll
      for (int p = 0; p < T::NP; ++p) {
        if (t < g.rows && v < dl_ld) {   // dl_ld is a multiple of 4
          ushort4 q = make_ushort4(out[0][p], out[1][p], out[2][p], out[3][p]);
          *reinterpret_cast<ushort4*>(dl + p * dl_plane + (long)t * dl_ld + v) = q;
        }
        if (t < dlt_ld)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e < g.count) dlt[p * dlt_plane + (long)(v + e) * dlt_ld + t] = out[e][p];
      }
    }
  }
  if (!dbias) return;
#pragma unroll
  for (int i = 0; i < T::TM; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float s = sums[i][e];
#pragma unroll
      for (int d = 1; d < 16; d *= 2) s += __shfl_xor(s, d, 64);
      const int v = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4 + e;
      if ((lane & 15) == 0 && v < g.count) dbias[(long)(tn * T::WN + wn) * g.classes + g.first + v] = s;
    }
}

__global__ __launch_bounds__(256) void k_loss_dbias(const float* __restrict__ parts, int count, int classes,
                                                    const float* __restrict__ ref, float* __restrict__ dbias) {
  const int v = blockIdx.x * 256 + threadIdx.x;
  if (v >= classes) return;
  float s = 0;
#pragma unroll 4
  for (int p = 0; p < count; ++p) s += parts[(long)p * classes + v];
  dbias[v] = s * *ref;
}

// out[n][m] = ref (sum_k A[m][k] B[n][k]): the gradient of a row n of W resp. h over its features m.
// kind 0: to fp32, 1: to bf16, both times ref; 2: to fp32 sums of a range of k (blockIdx.y), kept as
// they are, 3: added to what is there.
struct Product {
  void* out;
  long ld, split;        // elements between rows and between ranges of k
  int kind, k, per;      // k in all and per range
  const float* ref;
};
template <class T>
__global__ __launch_bounds__(T::THREADS) void k_loss_product(Operand a, Operand b, Product p, int tiles_m,
                                                             int tiles_n) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  int tm, tn;
  tile_of(tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  f32x4 acc[T::TM][T::TN] = {};
  const int k0 = blockIdx.y * p.per, k1 = k0 + p.per < p.k ? k0 + p.per : p.k;
  multiply<T>(a, b, 0, m0, n0, k0, k1, p.k, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % T::WM, wn = wave / T::WM;
  const float scale = p.kind < 2 ? *p.ref : 1.f;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const int n = n0 + (wn * T::TN + j) * 16 + (lane & 15);
    if (n >= b.rows) continue;
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      const int m = m0 + (wm * T::TM + i) * 16 + (lane >> 4) * 4;
      const long at = blockIdx.y * p.split + (long)n * p.ld + m;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (m + e >= a.rows) continue;
        const float v = acc[i][j][e] * scale;
        if (p.kind == 1) static_cast<uint16_t*>(p.out)[at + e] = bf16_bits(v);
        else if (p.kind == 3) static_cast<float*>(p.out)[at + e] += v;
        else static_cast<float*>(p.out)[at + e] = v;
      }
    }
  }
}

// Sums of the ranges of k -> gradient.
__global__ __launch_bounds__(256) void k_loss_sums(const float* __restrict__ sums, int count, long split,
                                                   long items, int bf16, const float* __restrict__ ref,
                                                   void* __restrict__ out) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long)gridDim.x * 256) {
    float s = 0;
    for (int q = 0; q < count; ++q) s += sums[q * split + i];
    s *= *ref;
    if (bf16) static_cast<uint16_t*>(out)[i] = bf16_bits(s);
    else static_cast<float*>(out)[i] = s;
  }
}

__global__ __launch_bounds__(256) void k_loss_zero(uint16_t* p, long items) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long)gridDim.x * 256) p[i] = 0;
}

unsigned grid_of(long items) {
  const long b = (items + 255) / 256;
  return (unsigned)(b < 1 ? 1 : b < 16384 ? b : 16384);
}

template <int NP>
using TileFor = Tile<128, 128, 2, 2, NP, NP == 1 ? 4 : 3>;
constexpr int kBM = 128, kBN = 128, kWN = 2;

// bf16 rows that the products can take where they lie: whole stages of features, 16-byte accesses.
bool direct(const LossArgs& a, const void* p, long stride) {
  return a.bf16 && a.features % 64 == 0 && stride % 8 == 0 && stride <= kMaxLd && ((uintptr_t)p & 15) == 0;
}

template <int NP>
Operand planes_of(const LossArgs& a, const void* src, long src_ld, int rows, char* to, int ld, hipStream_t st) {
  const long plane = (long)rows * ld;
  uint16_t* dst = reinterpret_cast<uint16_t*>(to);
  if (a.bf16)
    wino_launch((k_planes<uint16_t, NP>), dim3(grid_of(plane / 8)), dim3(256), st, (const uint16_t*)src, src_ld, rows,
                a.features, dst, (long)ld, plane);
  else
    wino_launch((k_planes<float, NP>), dim3(grid_of(plane / 8)), dim3(256), st, (const float*)src, src_ld, rows,
                a.features, dst, (long)ld, plane);
  return Operand{dst, ld, plane, 0, rows};
}

template <int NP>
Operand across(const LossArgs& a, const void* src, long src_ld, int rows, char* to, int ld,
               const int64_t* target, hipStream_t st) {
  const long plane = (long)a.features * ld;
  uint16_t* dst = reinterpret_cast<uint16_t*>(to);
  const dim3 grid((rows + 63) / 64, (a.features + 63) / 64);
  if (a.bf16)
    wino_launch((k_planes_across<uint16_t, NP>), grid, dim3(256), st, (const uint16_t*)src, src_ld, rows, a.features,
                dst, (long)ld, plane, target, a.ignore_index, a.classes);
  else
    wino_launch((k_planes_across<float, NP>), grid, dim3(256), st, (const float*)src, src_ld, rows, a.features, dst,
                (long)ld, plane, target, a.ignore_index, a.classes);
  return Operand{dst, ld, plane, 0, a.features};
}

const void* row_at(const LossArgs& a, const void* p, long row, long stride) {
  return static_cast<const char*>(p) + row * stride * (a.bf16 ? 2 : 4);
}

template <int NP>
hipError_t forward(const LossArgs& a, const void* h, const void* w, const float* bias, const int64_t* target,
                   float* loss, float* lse, char* ws, hipStream_t st) {
  typedef TileFor<NP> T;
  const LossLayout l = loss_layout(a, false);
  Operand oh = direct(a, h, a.h_stride) ? Operand{(const uint16_t*)h, a.h_stride, 0, 0, a.rows}
                                        : planes_of<NP>(a, h, a.h_stride, a.rows, ws + l.h, l.dp, st);
  float2* best = reinterpret_cast<float2*>(ws + l.parts);
  float* hit = reinterpret_cast<float*>(ws + l.target);
  const int tn = (a.rows + T::BN - 1) / T::BN;
  const bool as_is = direct(a, w, a.w_stride);
  // a launch holds fewer than 2^32 threads
  const long most = (1L << 22) / tn < 2 ? 2 * kBM : (1L << 22) / tn * kBM;
  const long piece = !as_is ? l.piece : a.classes < most ? a.classes : most;
  Logits g{bias, target, a.ignore_index, a.rows, a.classes, 0, 0, l.dp};
  int part = 0;
  for (long first = 0; first < a.classes; first += piece) {
    g.first = (int)first;
    g.count = (int)(a.classes - first < piece ? a.classes - first : piece);
    const void* rows = row_at(a, w, first, a.w_stride);
    const Operand ow = as_is ? Operand{(const uint16_t*)rows, a.w_stride, 0, 0, g.count}
                             : planes_of<NP>(a, rows, a.w_stride, g.count, ws + l.w, l.dp, st);
    const int tm = (g.count + T::BM - 1) / T::BM;
    wino_launch((k_loss_logits<T>), dim3(tm * tn), dim3(T::THREADS), st, ow, oh, g, tm, tn, part, best, hit);
    part += tm;
  }
  wino_launch(k_loss_join, dim3((a.rows + 15) / 16), dim3(256), st, (const float2*)best, part, (const float*)hit, g,
              loss, lse);
  return hipGetLastError();
}

template <int NP>
hipError_t backward(const LossArgs& a, const void* h, const void* w, const float* bias, const int64_t* target,
                    const float* lse, const float* dloss, void* dh, void* dw, float* dbias, char* ws,
                    hipStream_t st) {
  typedef TileFor<NP> T;
  const LossLayout l = loss_layout(a, true);
  float* ref = reinterpret_cast<float*>(ws + l.ref);
  Logits g{bias, target, a.ignore_index, a.rows, a.classes, 0, 0, l.dp};
  wino_launch(k_loss_weight, dim3(1), dim3(1024), st, dloss, g, ref);
  const Operand oh = direct(a, h, a.h_stride) ? Operand{(const uint16_t*)h, a.h_stride, 0, 0, a.rows}
                                              : planes_of<NP>(a, h, a.h_stride, a.rows, ws + l.h, l.dp, st);
  Operand ht{};
  if (dw) ht = across<NP>(a, h, a.h_stride, a.rows, ws + l.ht, l.tp, target, st);
  uint16_t* dl = reinterpret_cast<uint16_t*>(ws + l.dl);
  uint16_t* dlt = reinterpret_cast<uint16_t*>(ws + l.dlt);
  float* db = dbias ? reinterpret_cast<float*>(ws + l.dbias) : nullptr;
  float* sums = reinterpret_cast<float*>(ws + l.dh);
  const int tn = (int)((l.tp + T::BN - 1) / T::BN), td = (a.features + T::BM - 1) / T::BM;
  const bool as_is = direct(a, w, a.w_stride);
  const bool one = l.splits == 1 && l.piece >= a.classes;   // dh comes from one product
  for (long first = 0; first < a.classes; first += l.piece) {
    g.first = (int)first;
    g.count = a.classes - g.first < l.piece ? a.classes - g.first : l.piece;
    const int vp = (int)up(g.count, 64);
    const void* rows = row_at(a, w, first, a.w_stride);
    const Operand ow = as_is ? Operand{(const uint16_t*)rows, a.w_stride, 0, 0, g.count}
                             : planes_of<NP>(a, rows, a.w_stride, g.count, ws + l.w, l.dp, st);
    const int tm = (vp + T::BM - 1) / T::BM;
    const long dl_plane = (long)a.rows * vp, dlt_plane = (long)g.count * l.tp;
    wino_launch((k_loss_dlogits<T>), dim3(tm * tn), dim3(T::THREADS), st, ow, oh, g, tm, tn, lse, dloss,
                (const float*)ref, dl, (long)vp, dl_plane, dlt, (long)l.tp, dlt_plane, db);
    if (dh) {
      const Operand wt = across<NP>(a, rows, a.w_stride, g.count, ws + l.wt, vp, nullptr, st);
      const Operand od{dl, vp, dl_plane, 0, a.rows};
      const int per = (int)up((vp + l.splits - 1) / l.splits, 64);
      Product p{one ? dh : (void*)sums, a.features, (long)a.rows * a.features, one ? a.bf16 : first ? 3 : 2, vp, per,
                ref};
      const int t = (a.rows + T::BN - 1) / T::BN;
      wino_launch((k_loss_product<T>), dim3(td * t, l.splits), dim3(T::THREADS), st, wt, od, p, td, t);
    }
    if (dw) {
      const Operand od{dlt, l.tp, dlt_plane, 0, g.count};
      Product p{const_cast<void*>(row_at(a, dw, first, a.features)), a.features, 0, a.bf16, l.tp, l.tp, ref};
      const int t = (g.count + T::BN - 1) / T::BN;
      wino_launch((k_loss_product<T>), dim3(td * t), dim3(T::THREADS), st, ht, od, p, td, t);
    }
  }
  const long items = (long)a.rows * a.features;
  if (dh && !one)
    wino_launch(k_loss_sums, dim3(grid_of(items)), dim3(256), st, (const float*)sums, l.splits, items, items, a.bf16,
                (const float*)ref, dh);
  if (dbias)
    wino_launch(k_loss_dbias, dim3((a.classes + 255) / 256), dim3(256), st, (const float*)db, tn * T::WN, a.classes,
                (const float*)ref, dbias);
  return hipGetLastError();
}

}  // namespace

LossLayout loss_layout(const LossArgs& a, bool back) {
  LossLayout l{};
  const size_t T = (size_t)a.rows, D = (size_t)a.features, V = (size_t)a.classes;
  l.planes = a.bf16 ? 1 : 3;
  const size_t item = 2 * (size_t)l.planes;   // bytes of a value in planes
  l.dp = (int)up(D, 64);
  l.tp = (int)up(T, 64);
  // classes per piece: what the caller asks for, or as many as keep a piece's dl and weights, both
  // as rows and as columns, within 256 MiB
  size_t piece = a.piece ? (size_t)a.piece : ((size_t)256 << 20) / (2 * item * ((size_t)l.tp + l.dp));
  piece = up(piece < 1024 && !a.piece ? 1024 : piece, 256);
  if (piece > (size_t)kMaxLd) piece = (size_t)kMaxLd;
  l.piece = (int)(piece < V ? piece : V);
  const size_t P = (size_t)l.piece, vp = up(P, 64);
  size_t at = 0;
  const auto take = [&](size_t bytes) { const size_t was = at; at += up(bytes, 256); return was; };
  l.w = take(item * P * l.dp);
  l.h = take(item * T * l.dp);
  if (!back) {
    // a tile of classes never spans two pieces
    const size_t pieces = (V + P - 1) / P;
    l.parts = take(8 * T * (pieces * ((P + kBM - 1) / kBM) + (V + kBM - 1) / kBM));
    l.target = take(4 * T);
    l.splits = 1;
  } else {
    l.ref = take(4);
    l.ht = take(item * D * l.tp);
    l.wt = take(item * D * vp);
    l.dl = take(item * T * vp);
    l.dlt = take(item * P * l.tp);
    // ranges of classes until dh's tiles fill the chip, each of 512 classes or more
    const size_t tiles = ((D + kBM - 1) / kBM) * ((T + kBN - 1) / kBN);
    size_t s = tiles ? (256 + tiles - 1) / tiles : 1;
    if (s > vp / 512) s = vp / 512;
    if (s < 1) s = 1;
    l.splits = (int)s;
    l.dh = take(4 * T * D * s);
    l.dbias = take(4 * V * kWN * ((l.tp + kBN - 1) / kBN));
  }
  l.bytes = at ? at : 256;
  return l;
}

hipError_t launch_loss(const LossArgs& a, const void* h, const void* w, const float* bias,
                       const int64_t* target, float* loss, float* lse, char* ws, hipStream_t st) {
  return a.bf16 ? forward<1>(a, h, w, bias, target, loss, lse, ws, st)
                : forward<3>(a, h, w, bias, target, loss, lse, ws, st);
}

hipError_t launch_loss_backward(const LossArgs& a, const void* h, const void* w, const float* bias,
                                const int64_t* target, const float* lse, const float* dloss, void* dh,
                                void* dw, float* dbias, char* ws, hipStream_t st) {
  if (a.rows == 0) {   // no rows: the weights' gradient is zero
    const long items = (long)a.classes * a.features * (a.bf16 ? 1 : 2);
    if (dw) wino_launch(k_loss_zero, dim3(grid_of(items)), dim3(256), st, (uint16_t*)dw, items);
    if (dbias)
      wino_launch(k_loss_zero, dim3(grid_of(2L * a.classes)), dim3(256), st, (uint16_t*)dbias, 2L * a.classes);
    return hipGetLastError();
  }
  return a.bf16 ? backward<1>(a, h, w, bias, target, lse, dloss, dh, dw, dbias, ws, st)
                : backward<3>(a, h, w, bias, target, lse, dloss, dh, dw, dbias, ws, st);
}

}  // namespace wino
