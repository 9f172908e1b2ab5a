// Blocks of the layer norm's gradient and the tiles' way round the pairs of the head's products: arithmetic on sizes alone, so
// that a host without a device can check it.
#pragma once

#include <algorithm>
#include <cstdint>

#ifdef __CUDACC__
#define PRM_HOST_DEVICE __host__ __device__
#else
#define PRM_HOST_DEVICE
#endif

namespace prm {

// The gradient's blocks: every group of rows has `parts` of them, as many as are resident together.  The sizes
// do not depend on the device, so that the scratch's do not either.
inline int64_t layernorm_parts_most(int64_t cols) {
  return cols <= 256 ? 444 : cols <= 512 ? 592 : cols <= 1024 ? 1184 : cols <= 2048 ? 592 : cols <= 4096 ? 296 : 148;
}
// Rows that start anywhere need 8 | parts * (rows per block and turn), or a turn for all rows, so that all
// rows of a thread start alike: up to 8 parts.
inline int64_t layernorm_parts_bound(int64_t rows_per_group, int64_t groups, int64_t cols) {
  return std::min(rows_per_group, std::max<int64_t>(8, layernorm_parts_most(cols) / groups));
}
inline int64_t layernorm_parts(int64_t rows_per_group, int64_t groups, int64_t cols, int rows_per_turn, int blocks,
                               bool shift) {
  const int64_t turns = (rows_per_group + rows_per_turn - 1) / rows_per_turn;
  int64_t parts = std::max<int64_t>(1, std::min<int64_t>(blocks, layernorm_parts_most(cols)) / groups);
  // a block has two rows before more than an SM's worth of blocks have one: each leaves a line to add
  parts = std::min(parts, std::max<int64_t>((148 + groups - 1) / groups, turns / 2));
  if (shift) {
    const int64_t unit = rows_per_turn >= 8 ? 1 : 8 / rows_per_turn;
    parts = std::max(unit, parts / unit * unit);
  }
  return std::min(parts, turns);
}

// The i-th tile of a pair in a launch of one product (t1 = 0) or two that do not depend on one another; false if it has none
// left.  The first one's tiles go round the pairs; those that its last round leaves idle take `extra` tiles of the second for it,
// as many as take as long as one of the first; then the second's rest goes round.
PRM_HOST_DEVICE inline bool pair_tile(int t0, int t1, int extra, int pair, int pairs, int i, int& which, int& tile) {
  which = 0;
  tile = pair + i * pairs;
  if (tile < t0) return true;
  which = 1;
  const int used = t0 % pairs, own = used > 0 && pair >= used ? extra : 0;
  i -= t0 / pairs + (pair < used);
  tile = i < own ? (pair - used) * extra + i : (used > 0 ? (pairs - used) * extra : 0) + pair + (i - own) * pairs;
  return tile < t1;
}

}  // namespace prm
