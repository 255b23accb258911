// Where the products (wino_products.hpp) read an operand of fp32 values that lies in a caller's tensor, k
// along its rows.  A stage is 32 k, a line of 128 bytes; rows have any length, so the last stage of a row
// may be a part of one, and behind the operand's last row lies memory that is not the tensor's.
//
// A buffer access is refused by its lane's offset; how the scalar offset enters that check is not relied
// on: it counts only in stages that lie in the row, whose every byte is the operand's, or is refused by
// the lane's row alone.  In a part of a stage k stands in the lane's offset, and 16-byte pieces that begin
// behind the row are refused.  What then passes the end of the last row is cut off by the descriptor's
// size, to the byte; what passes the end of another row is masked by the reader.
#pragma once
#include <hip/hip_runtime.h>

namespace wino {
namespace prod {

constexpr int kRefused = 0x40000000;   // an offset beyond every such operand's tile

// Stages cover `cols` k: none lies behind a row.
__host__ __device__ inline int whole_stages_of_32(int cols) { return (cols + 31) / 32 * 32; }

// The first of four values that a lane of a copy of eight rows takes to its place, in a stage: the pieces
// of a row change places by the row.
__host__ __device__ inline int copied_value(int lane) { return ((lane & 7) ^ (lane >> 3)) * 4; }
// Of the two pieces that a lane of a 32 x 32 tile's load reads.
__host__ __device__ inline int loaded_value(int lane, int piece) { return (lane >> 4) * 8 + piece * 4; }

struct Source {
  int lane, scalar;   // bytes
};
// `at`: the lane's place in the stage at k = 0, bytes; value: the stage's k there.
__host__ __device__ inline Source source_at(int at, int value, int k, int cols) {
  if (k + 32 <= cols) return {at, k * 4};
  return {k + value < cols ? at + k * 4 : kRefused, 0};
}

}  // namespace prod
}  // namespace wino
