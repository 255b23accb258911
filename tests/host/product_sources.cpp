// The addresses at which the products read a caller's fp32 tensor along its rows: every tile of 64 and 32
// rows, every lane and stage, against the tensor's end.  A descriptor's range check is taken in three ways,
// by the lane's offset alone and by its sum with the scalar one before and after a wrap below zero: under
// each no byte behind the tensor is read, and every value of the tensor is.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "wino_product_sources.hpp"

using namespace wino::prod;

static long reads = 0;

static bool passes(int check, unsigned lane, unsigned scalar, unsigned size) {
  if (check == 0) return lane < size;
  if (check == 1) return (unsigned long)lane + scalar < size;
  return lane < size - scalar;   // as hardware of 32 bits would subtract
}

// One tile: `side` rows from `first`; f(lane, i, &row, &value) names a lane's i-th piece.
template <class F>
static void tile(int rows, int cols, int ld, int first, int side, int pieces, F&& f) {
  const int left = std::min(rows - first, side);
  const unsigned size = ((left - 1) * (long)ld + cols) * 4;
  const long end = ((long)(rows - 1) * ld + cols - (long)first * ld) * 4;   // of the tensor, from the tile's start
  for (int check = 0; check < 3; ++check) {
    std::vector<char> seen((size_t)left * cols);
    for (int k = 0; k < whole_stages_of_32(cols); k += 32)
      for (int lane = 0; lane < 64; ++lane)
        for (int i = 0; i < pieces; ++i) {
          int row, value;
          f(lane, i, row, value);
          const Source s = source_at((row * ld + value) * 4, value, k, cols);
          for (int e = 0; e < 4; ++e, ++reads) {
            if (!passes(check, s.lane + 4 * e, s.scalar, size)) continue;
            const long at = (long)s.lane + s.scalar + 4 * e;
            if (at + 4 > end) {
              std::printf("rows %d cols %d ld %d first %d side %d k %d lane %d check %d: byte %ld of %ld\n", rows, cols, ld,
                          first, side, k, lane, check, at, end);
              std::exit(1);
            }
            if (row < left && k + value + e < cols && at == ((long)row * ld + k + value + e) * 4)
              seen[(size_t)row * cols + k + value + e] = 1;
          }
        }
    if (std::count(seen.begin(), seen.end(), 1) != (long)seen.size()) {
      std::printf("rows %d cols %d ld %d first %d side %d check %d: not all values read\n", rows, cols, ld, first, side, check);
      std::exit(1);
    }
  }
}

int main() {
  for (int rows : {1, 2, 7, 16, 17, 31, 32, 33, 64, 65, 66, 96, 97})
    for (int cols : {1, 2, 3, 4, 5, 8, 13, 28, 29, 31, 32, 33, 36, 60, 63, 64, 65, 67, 92, 93, 96, 97, 128, 130, 515, 925})
      for (int more : {0, 1, 3, 8, 100}) {
        const int ld = cols + more;
        for (int first = 0; first < rows; first += 64)   // copies of eight rows
          tile(rows, cols, ld, first, 64, 8, [](int lane, int i, int& row, int& value) {
            row = i * 8 + (lane >> 3), value = copied_value(lane);
          });
        for (int first = 0; first < rows; first += 32)   // two pieces of two blocks of sixteen rows
          tile(rows, cols, ld, first, 32, 4, [](int lane, int i, int& row, int& value) {
            row = (i >> 1) * 16 + (lane & 15), value = loaded_value(lane, i & 1);
          });
      }
  std::printf("ok %ld\n", reads);
  return 0;
}
