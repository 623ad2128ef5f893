// Chunks of eight neighbours of many rows, one behind the other: how kernels without sums over a row share a matrix among threads.
#pragma once

#include "operators.h"

namespace gan {

// Chunks are numbered row by row, `eights` to a row.  A block takes `TILE` neighbouring chunks at a time, so that no width leaves threads without work; which row a
// chunk is in follows from the tile's first row (a division for the whole wave) and, within the tile, a product.
struct RowChunks {
  long long rows;
  unsigned eights;                                                // chunks of a row
  unsigned inverse;                                               // 2^32 / eights rounded up (rows of 2 to TILE chunks)
};

constexpr unsigned MOST_TILE = 4096;                              // chunks of a tile

inline RowChunks row_chunks(long long rows, int cols) {
  const unsigned eights = (unsigned)(((long long)cols + 7) / 8);
  return {rows, eights, 0xffffffffu / eights + 1};
}
// blocks of a launch: tiles beyond them are taken in turns (a launch has fewer than 2^32 threads)
inline unsigned chunk_blocks(const RowChunks& s, int tile, unsigned most) {
  const long long tiles = (s.rows * s.eights + tile - 1) / tile;
  return (unsigned)(tiles < most ? tiles : most);
}

// chunk `t` behind chunk `col` of row `row`; t < TILE <= MOST_TILE: below 2^24 the product is exact
__device__ __forceinline__ void chunk_at(const RowChunks& s, long long row0, unsigned col0, unsigned t, long long& row, unsigned& chunk) {
  const unsigned c = col0 + t;
  const unsigned down = s.eights > MOST_TILE ? (c >= s.eights ? 1u : 0u) : s.eights == 1 ? c : __umulhi(c, s.inverse);
  row = row0 + down;
  chunk = c - down * s.eights;
}

}  // namespace gan
