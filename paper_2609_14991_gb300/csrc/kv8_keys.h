// Which keys of the 8-bit paged cache a tile of query rows sees, and how they are dealt
// out to CTAs (kv8_rows.cu, kv8_tiles.cu); how many CTAs an append takes (kv8.cu).
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define TSD_HD __host__ __device__
#else
#define TSD_HD
#endif

namespace tsd {

constexpr int kKv8Unit = 16;  // tokens that are sure to share a block

// The units of keys that rows at positions pos0 .. pos1 see: first those of the
// sinks before the window, then the window's.
struct KeyTiles {
  int sink, from, total;  // units 0 .. sink-1, then units from, from + 1, ..
  TSD_HD int token(int j) const { return kKv8Unit * (j < sink ? j : from + j - sink); }
};
TSD_HD inline KeyTiles key_tiles(int pos0, int pos1, int window, int sinks) {
  const int first = window > 0 && pos0 >= window ? pos0 - window + 1 : 0;
  KeyTiles k;
  k.sink = ((sinks < first ? sinks : first) + kKv8Unit - 1) / kKv8Unit;
  k.from = k.sink > first / kKv8Unit ? k.sink : first / kKv8Unit;
  k.total = k.sink + pos1 / kKv8Unit + 1 - k.from;
  return k;
}

// Where share i of `parts` even shares of `all` begins.
TSD_HD inline int share_from(int all, int i, int parts) {
  const int each = all / parts, left = all - each * parts;
  return i * each + (i < left ? i : left);
}

// Split `split`'s share of `units` units: its first key tile (tile_units each), its key
// tiles, and the steps (step_units each) that they take.
struct KeyShare {
  int lo, n, steps;
};
TSD_HD inline KeyShare key_share(int units, int tile_units, int step_units, int split, int splits) {
  const int all = (units + tile_units - 1) / tile_units;
  KeyShare s;
  s.lo = share_from(all, split, splits);
  s.n = share_from(all, split + 1, splits) - s.lo;
  const int from = s.lo * tile_units, to = from + s.n * tile_units, end = units < to ? units : to;
  s.steps = end > from ? (end - from + step_units - 1) / step_units : 0;  // (an empty share begins past the last unit)
  return s;
}

// Blocks of a sequence that an append's launch has CTAs for (a CTA takes more in turn): all that
// max_new rows may touch; one row's without starts; else sixteen times the mean's, so that a launch
// grows with its rows and sequences and not with their product (1024 x 1, 8 heads of 128: 65 us, with
// CTAs for all rows in each 168; a prompt of 4000 beside 63 x 1: 25 and 41).
inline int64_t append_blocks(int n, int rows, bool starts, int max_new, int block) {
  const int64_t mean = ((int64_t)rows + n - 1) / n;
  const int64_t most = max_new ? max_new : !starts ? 1 : 16 * mean;
  return ((most < rows ? most : rows) + 2 * block - 2) / block;
}

}  // namespace tsd
