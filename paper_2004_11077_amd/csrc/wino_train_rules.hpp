// What the operators of a training step run on: which tiles, how many ranges of k or of rows, and from that the
// regions of their workspaces.  Host arithmetic only.
#pragma once
#include "wino_train.hpp"

namespace wino {
namespace prod {

constexpr long kMaxLd = 1L << 21;   // elements between rows: 256 rows of it are 2^30 bytes

// Share of the 256 x 256 tiles' rate that other tiles reach when nothing is idle (16384 x 2048 x 4096 in bf16:
// 1421 TFLOP/s and 1297; two planes, 13824 x 512 x 512: 128 x 128 tiles 22.2 us with 0.84 of the chip at work,
// 64 x 64 ones 25.6 us with 0.96).
inline double rate_of(int side) { return side == 256 ? 1.0 : side == 128 ? 0.92 : 0.8; }
// Side of the square tiles (256, 128 or 64) for `z` products of m x n: the one that leaves least of the
// chip idle, counting what of its tiles lies outside, and compute units that wait for the others' last tile.
// (X of 6144 x 1536, k of 1536: 128 x 128 tiles 130 us, 64 x 64 ones 123; of 3 x 4608 x 512, k of 512: 33.5
// and 39.)
inline int side_for(double m, double n, double z) {
  int best = 64;
  double most = 0;
  for (int side = 256; side >= 64; side /= 2) {
    const double tiles = __builtin_ceil(m / side) * __builtin_ceil(n / side) * z;
    const double score = rate_of(side) * m * n * z / (__builtin_ceil(tiles / 256) * 256 * side * side);
    if (score > most) most = score, best = side;
  }
  return best;
}
inline long count_of(long m, long n, long side) { return ((m + side - 1) / side) * ((n + side - 1) / side); }

}  // namespace prod

// ---- linear cross entropy --------------------------------------------------------------------
namespace loss {

using namespace prod;

constexpr int kRange = 256;        // partial maxima of a tensor
// Numbers that kernels hand to later ones.
struct Numbers {
  float ref;              // largest finite |dloss|, one where that is zero
  int of_w, of_h;         // exponents of W's, h's planes: they hold 2^e times the values
  float max_w[kRange], max_h[kRange];
};

// Products with k along the rows of both operands, over k of them: 32 x 32 with k shared by the waves where
// there are few tiles, which for fp32, three or six products a term, are more, and more again where half
// of a tile of 64 or more would be empty.  (Training steps: 64 x 512 x 2048 in fp32 56 us, with tiles of 64 62;
// 4330 x 3610 x 8, 68 tiles: 178 and 251; 4096 x 2048 x 128, 128 tiles: 191 and 169; 3 x 925 x 10000, 157 tiles: 67
// and 95; 900 x 4092 x 401 in bf16, 105 tiles: 128 and 104.)
constexpr long few_tiles(bool bf16) { return bf16 ? 64 : 128; }
inline int least_side(bool bf16, long m, long n, long k) {
  const long few = !bf16 && (m <= 32 || n <= 32) ? 256 : few_tiles(bf16);
  return count_of(m, n, 64) < few && k >= 256 ? 32 : 64;
}
inline int side_along(bool bf16, long m, long n, long k) {
  const int side = side_for(m, n, 1);
  return side == 64 ? least_side(bf16, m, n, k) : side;
}
constexpr int waves_n(int side) { return side == 256 ? 4 : 2; }

// fp32 as it stands: few rows or classes, where the time is the passage of W or h through memory (75113 x 925 and 3 rows, a
// training step: 324 us, by way of planes 821; 192 rows 907 and 1149, 256 rows 1160 and 1237; 256 x 1024 x
// 8192, where every tile of W is cut four times: 151 and 143; 44 x 1452 x 2481: 70 and 97; 20000 x 1030 x 3: 228 and 299; 4096 x 2048 x 128: 197 and 169).  Values below 2^-102
// lose lower pieces to bf16's smallest numbers there, which planes keep, so small tensors, where the gain is
// a few microseconds of launches (64 x 64 x 1000: 42.3 us and 45.2), stay with the planes.
inline bool as_it_stands(const LossArgs& a) {
  const double least = 1 << 16;
  return !a.bf16 && a.h_stride <= kMaxLd / 2 && a.w_stride <= kMaxLd / 2 &&
         ((a.rows <= 192 && (double)a.features * a.classes >= least) ||
          (a.classes <= 64 && (double)a.features * a.rows >= least));
}

// Tiles of `count` classes: of the logits in the forward pass, and of dW.
inline int logits_side(const LossArgs& a, const LossLayout& l, long count) {
  return as_it_stands(a) ? least_side(false, count, a.rows, l.dp) : side_along(a.bf16, count, a.rows, l.dp);
}
inline int dw_side(const LossArgs& a, const LossLayout& l, long count) {
  return l.dw_splits > 1 || as_it_stands(a) ? 64 : side_for(count, a.features, 1);
}

}  // namespace loss

inline LossLayout loss_layout(const LossArgs& a, bool back) {
  using namespace loss;
  LossLayout l{};
  const size_t T = (size_t)a.rows, D = (size_t)a.features, V = (size_t)a.classes;
  const int np = a.bf16 ? 1 : 2;
  const size_t item = 2 * (size_t)np;   // bytes of a value in planes
  l.dp = (int)up(D, 64);
  // classes per piece: what the caller asks for, or as many as keep a piece's dl, and its planes of W if
  // it may need them, within 256 MiB
  const size_t most = T > (size_t)l.dp || as_it_stands(a) ? T : (size_t)l.dp;
  size_t piece = a.piece ? (size_t)a.piece : ((size_t)256 << 20) / (item * (most ? most : 1));
  piece = up(piece < 1024 && !a.piece ? 1024 : piece, 256);
  if (piece > (size_t)kMaxLd / 2) piece = (size_t)kMaxLd / 2;   // rows of dl on two planes
  l.piece = (int)(piece < V ? piece : V);
  const size_t P = (size_t)l.piece, vp = up(P, 64);
  size_t at = 0;
  const auto take = [&](size_t bytes) { const size_t was = at; at += up(bytes, 256); return was; };
  l.numbers = take(sizeof(Numbers));
  if (!as_it_stands(a)) l.w = take(item * P * l.dp);
  l.h = take(item * T * l.dp);
  l.splits = 1;
  if (!back) {
    // pieces are whole multiples of 256 classes, so no tile spans two
    // of side_along() for any classes (32 or fewer are one tile of either side)
    const size_t least = T >= 64 * (size_t)few_tiles(a.bf16) ? 64 : 32;
    l.parts = take(8 * T * (up(V, 256) / least));
    l.target = take(4 * T);
    l.unit_w = take(4 * P);
    l.unit_h = take(4 * T);
  } else {
    l.dl = take(item * T * vp);
    // bf16: with few rows a gradient may be one term of dl, whose rounding is then as large as the result's; with
    // few of them, or little to do, dl is kept on two bf16 values
    l.two = a.bf16 && (T <= 64 || (double)T * D * V <= 1 << 30);
    if (l.two) l.rest = take(item * T * vp);
    const bool stands = as_it_stands(a);
    l.side = stands ? least_side(false, (long)P, (long)T, l.dp) : side_along(a.bf16, (long)P, (long)T, l.dp);
    // ranges of classes, each of 512 or more, until dh's tiles fill the chip: one tile of 256 a compute
    // unit, or two of the smaller ones
    const long room = (long)(vp / 512 ? vp / 512 : 1);
    double most = 0;
    for (int side = stands ? 64 : 256; side >= 64 && T; side /= 2) {
      const long tiles = count_of((long)D, (long)T, side), slots = side == 256 ? 256 : 512;
      long ranges = slots / tiles;
      ranges = ranges > room ? room : ranges < 1 ? 1 : ranges;
      const double score = rate_of(side) * D * T * ranges / ((double)((tiles * ranges + 255) / 256) * 256 * side * side);
      if (score > most) most = score, l.dh_side = side, l.splits = (int)ranges;
    }
    if (l.splits > 64) l.splits = 64;   // k_loss_sums adds them up one after the other
    l.dh = take(4 * T * D * l.splits);
    // ranges of rows, each of 256 or more, where dW has few tiles of 64 (a training step of 2048 x 64 x 1000 in
    // fp32: 63 us, without them 87)
    const long tiles = count_of((long)P, (long)D, 64);
    long ranges = tiles < 128 ? 256 / tiles : 1;
    if (ranges > (long)T / 256) ranges = (long)T / 256;
    l.dw_splits = (int)(ranges < 1 ? 1 : ranges > 64 ? 64 : ranges);
    if (l.dw_splits > 1) l.dw = take(4 * P * D * l.dw_splits);
    l.dbias = take(4 * V * waves_n(l.side) * (T ? (T + l.side - 1) / l.side : 1));
  }
  l.bytes = at;
  return l;
}

// ---- orthogonalised updates ------------------------------------------------------------------
namespace update {

using namespace prod;

constexpr int kNormParts = 256;    // partial sums of a matrix's squares

inline int tiles_of(int side, int tile) { return (side + tile - 1) / tile; }
inline int half_of(int tiles) { return tiles * (tiles + 1) / 2; }

// Symmetric products of few tiles and not many k: no barriers, one launch.  (A of 4 x 64 rows, k of 576: 8.4
// us, and 9.5 in four ranges with their join; of 3 x 256 rows, k of 2304: 20.9 us and 18.9.)
inline bool few(const UpdateLayout& l, int batch, int k) { return (long)l.r * l.r * batch <= 256L * 256 * 4 && k <= 1024; }
// Tiles of X.
inline int next_side(const UpdateLayout& l, int batch) { return side_for(l.c, l.r, batch); }

}  // namespace update

inline UpdateLayout update_layout(const UpdateArgs& a) {
  using namespace update;
  UpdateLayout l{};
  l.r = a.rows < a.cols ? a.rows : a.cols;
  l.c = a.rows < a.cols ? a.cols : a.rows;
  l.rp = (int)up(l.r, 64);
  l.cp = (int)up(l.c, 64);
  size_t at = 0;
  const auto take = [&](size_t bytes) { const size_t was = at; at += up(bytes, 256); return was; };
  const size_t item = 2 * 2 * (size_t)a.batch;   // two planes
  l.norms = take(sizeof(double) * kNormParts * a.batch);
  l.x = take(item * l.r * l.cp);
  l.x2 = take(item * l.r * l.cp);
  l.gram = take(item * l.r * l.rp);
  l.poly = take(item * l.r * l.rp);
  l.splits = 1;
  if (a.batch && l.r && !few(l, a.batch, (int)up(l.c, 32))) {
    // ranges of A's k until its tiles fill the chip, each of 512 or more
    l.side = (long)half_of(tiles_of(l.r, 128)) * a.batch >= 64 ? 128 : 64;
    const long tiles = (long)half_of(tiles_of(l.r, l.side)) * a.batch;
    long s = (512 + tiles / 2) / tiles;
    if (s > l.cp / 512) s = l.cp / 512;
    l.splits = (int)(s < 1 ? 1 : s);
    if (l.splits > 1) l.parts = take(4 * (size_t)l.splits * a.batch * l.r * l.rp);
  }
  l.bytes = at ? at : 256;
  return l;
}

}  // namespace wino
