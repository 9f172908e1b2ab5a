// Blocks of the layer norm's gradient, pieces and splits of the head's gradient, and the tiles' way round the pairs of the head's
// products: arithmetic on sizes alone, so that a host without a device can check it.
#pragma once

#include <algorithm>
#include <cstddef>
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

// The lines of a group that the scratch holds: with whole octs only what resident blocks leave (1024 groups of 8 rows x 8192: 64
// MB, with 8 lines 512 MB).  Such rows that all the same start unlike one another, and would need more, go to the kernel of single
// elements, for which any number will do.
inline int64_t layernorm_lines(int64_t rows_per_group, int64_t groups, int64_t cols) {
  if (cols % 8 != 0) return layernorm_parts_bound(rows_per_group, groups, cols);
  return std::min(rows_per_group, std::max<int64_t>(1, layernorm_parts_most(cols) / groups));
}
// Lines of a group that one thread per column adds; more are added by a block per 32 columns.
constexpr int kLinesPerThread = 16;
// Whether the gradient's grids, of its blocks and of those that add their lines, fit a launch: with up to 2^30 - 1 groups, unless
// rows are very wide as well.
inline bool layernorm_grids_ok(int64_t rows_per_group, int64_t groups, int64_t cols) {
  const int64_t parts = layernorm_parts_bound(rows_per_group, groups, cols), width = parts > kLinesPerThread ? 32 : 256;
  return groups * parts <= 0x7fffffffLL && groups * ((cols + width - 1) / width) * 2 <= 0x7fffffffLL;
}

constexpr int kHeadTile = 256;                   // edge of the head's tiles
constexpr int kHeadStage = 128;                  // k that a stage of a tile's main loop holds

inline int64_t ceil_to(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }

// The head's gradient: pieces of the vocabulary whose G fits 512 MB, of alike width but for the last, which may have a few columns
// only (pieces that stay in the L2, 64 MB, leave each product too few tiles: 8192 x 64 x 32768 takes 729 us with them, 470 with
// one piece), and grad_x's sums: parts of one product's k where there are few tiles, the pieces' running sums where there are
// several.
struct HeadGradPlan {
  int64_t piece, ld_g, ld_part;
  int pieces, split;
  size_t g_bytes, part_bytes;
};
inline HeadGradPlan head_grad_plan(int64_t n, int64_t d, int64_t vocab) {
  HeadGradPlan p;
  const int64_t most = std::max<int64_t>(2048, ((int64_t)512 << 20) / (2 * n) / kHeadTile * kHeadTile);
  p.pieces = (int)((vocab + most - 1) / most);
  p.piece = ceil_to((vocab + p.pieces - 1) / p.pieces, kHeadTile);
  p.pieces = (int)((vocab + p.piece - 1) / p.piece);
  p.ld_g = ceil_to(std::min(p.piece, vocab), 64);
  const int64_t tiles = ((n + kHeadTile - 1) / kHeadTile) * ((d + kHeadTile - 1) / kHeadTile);
  const int64_t stages = (std::min(p.piece, vocab) + kHeadStage - 1) / kHeadStage;
  p.split = (int)std::max<int64_t>(1, std::min<int64_t>({74 / tiles, stages / 4, 16}));
  p.ld_part = ceil_to(d, 4);
  p.g_bytes = (size_t)ceil_to(n * p.ld_g * 2, 256);
  p.part_bytes = p.pieces > 1 || p.split > 1 ? (size_t)p.split * n * p.ld_part * 4 : 0;
  return p;
}
// Parts of k for a piece of `wide` columns: the plan's, but none without a stage, whose tiles would wait for sums that nobody
// computes.  The first piece has them all; where the last one has fewer, the other parts keep the sums of the pieces before it.
inline int head_grad_split(const HeadGradPlan& p, int64_t wide) {
  return (int)std::min<int64_t>(p.split, (wide + kHeadStage - 1) / kHeadStage);
}
// The stages s0 .. s1 - 1 of part `at` of `split`.
PRM_HOST_DEVICE inline void head_part(int stages, int split, int at, int& s0, int& s1) {
  s0 = (int)((int64_t)stages * at / split);
  s1 = (int)((int64_t)stages * (at + 1) / split);
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
