// 8-bit rows with a power-of-two scale per 32 elements: where a scale lies and how it is made.
#pragma once

#include "jk_paged.cuh"

#define MX_BLOCK 32                       // elements of a row that share a scale
#define MX_TILE_BYTES 512                 // scales of 128 rows x 4 blocks

// Byte of the scale of row r, block k, in tiles of 128 rows x 4 blocks; k_tiles = ceil(n / 128).
__host__ __device__ inline size_t mx_scale_at(size_t r, int k, int k_tiles) {
  return ((r >> 7) * (size_t)k_tiles + (size_t)(k >> 2)) * MX_TILE_BYTES + (r & 31) * 16 + ((r & 127) >> 5) * 4 +
         (size_t)(k & 3);
}
static inline int mx_k_tiles(int64_t n) { return (int)((n + 127) / 128); }

// Do [a, a + na) and [b, b + nb) share a byte?
static inline bool jk_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + nb && y < x + na;
}

// The same for rows of wa and wb bytes, each sa and sb bytes behind the last: rows of one stride may lie between one
// another, as the columns of one buffer do.
static inline bool jk_rows_overlap(const void* a, size_t rows_a, size_t wa, size_t sa, const void* b, size_t rows_b,
                                   size_t wb, size_t sb) {
  if (!jk_overlap(a, (rows_a - 1) * sa + wa, b, (rows_b - 1) * sb + wb)) return false;
  if (sa != sb) return true;
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  const size_t off = y >= x ? (y - x) % sa : (sa - (x - y) % sa) % sa;      // columns from a's first to b's first
  return off < wa || off + wb > sa;
}
