// How the work of a mixture-of-experts layer's products is cut into equal shares, for kernels and for the tests of host code.
#pragma once

#include <cstdint>

#include "layer_internal.h"

#ifndef SK_BOTH
#if defined(__HIPCC__)
#define SK_BOTH __host__ __device__ __forceinline__
#else
#define SK_BOTH inline
#endif
#endif

namespace sk {
namespace moe {

SK_BOTH int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// Rows of activations that a tile is made for.
SK_BOTH int32_t mode_of(int32_t rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : 32; }
// Rows of weights that a tile has: 16 of two matrices; of one 16 for up to 8 rows of activations, and 32 for more (whose loads, from another compute
// unit's reach, would be twice those of the weights).
SK_BOTH constexpr int32_t rows_of_tile(int32_t matrices, int32_t mode) { return matrices == 1 && mode > 8 ? 32 : 16; }
SK_BOTH int32_t tiles_of(int32_t rows, int32_t matrices, int32_t mode) {
  const int32_t t = rows_of_tile(matrices, mode);
  return rows / t + (rows % t != 0);
}
// All tiles of a launch stand in a row, each as long as it takes: the loads of a wave, and some for its beginning and end.  k_len: elements of its
// reduction, `matrices` of weights, `parts` of the activations (their planes of as many bytes as 16-bit numbers).
constexpr int32_t EXTRA = 8;
SK_BOTH int64_t cost(int32_t k_len, int32_t matrices, int32_t parts, int32_t mode) {
  return (int64_t)((k_len + 255) / 256) * (matrices * rows_of_tile(matrices, mode) / 8 + parts * mode / 8) + EXTRA;
}

// A workgroup has the tiles that begin in its share.
struct Share {
  int64_t begin, end;
};
SK_BOTH Share share_of(int64_t total, int64_t shares, int64_t i) { return Share{total * i / shares, total * (i + 1) / shares}; }
// All tiles of a group stand side by side.  The first tile that begins at or behind a place: group g is the last that begins at or before it (at
// `begin`, with `tiles` tiles of `each`); tile == tiles: the first of the next group.
SK_BOTH int32_t tile_from(int64_t at, int64_t begin, int64_t each, int32_t tiles) { return (int32_t)least(tiles, (at - begin + each - 1) / each); }

}  // namespace moe
}  // namespace sk
