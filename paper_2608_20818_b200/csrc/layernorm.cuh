// Layer norm with the residual's addition and dropout: what its two directions share.
#pragma once

#include "dropout.cuh"

namespace prm {

// Scale and shift of a row: one row of them for all rows, or one for each group of `rows_per_group`.
struct Affine {
  const void* weight;      // may be null (1)
  const void* bias;        // may be null (0)
  int64_t ld_w, ld_b;
  int fp32;
  int add_one;             // the weight is 1 + what is stored
};

__device__ __forceinline__ void affine_weight(const Affine& a, int64_t group, int first, int cols, float2 (&w)[4]) {
  if (!a.weight) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = make_float2(1.f, 1.f);
    return;
  }
  const char* p = reinterpret_cast<const char*>(a.weight) + group * a.ld_w * (a.fp32 ? 4 : 2);
  load_factors(p, a.fp32, first, cols, w);
  if (a.add_one) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = add2(w[e], make_float2(1.f, 1.f));
  }
}
__device__ __forceinline__ void affine_bias(const Affine& a, int64_t group, int first, int cols, float2 (&b)[4]) {
  if (!a.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = make_float2(0.f, 0.f);
    return;
  }
  const char* p = reinterpret_cast<const char*>(a.bias) + group * a.ld_b * (a.fp32 ? 4 : 2);
  load_factors(p, a.fp32, first, cols, b);
}
__device__ __forceinline__ float affine_weight1(const Affine& a, int64_t group, int c) {
  if (!a.weight) return 1.f;
  const float w = load1(a.weight, a.fp32, group * a.ld_w + c);
  return a.add_one ? 1.f + w : w;
}
__device__ __forceinline__ float affine_bias1(const Affine& a, int64_t group, int c) {
  return a.bias ? load1(a.bias, a.fp32, group * a.ld_b + c) : 0.f;
}

// Zeros for the oct's elements outside the row.
__device__ __forceinline__ void clear_outside(int first, int cols, float2 (&v)[4]) {
  if (first < 0 || first + 8 > cols) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (first + 2 * k < 0 || first + 2 * k >= cols) v[k].x = 0.f;
      if (first + 2 * k + 1 < 0 || first + 2 * k + 1 >= cols) v[k].y = 0.f;
    }
  }
}

inline bool layernorm_ld_ok(int64_t ld) { return ld >= 0 && ld <= ((int64_t)1 << 40); }

// The gradient's blocks: every group of rows has `parts` of them.  256 threads up to 2048 columns (a
// thread holds an oct of a row), else a block to one or two rows.  The sizes do not depend on the device,
// so that the scratch's do not either.
inline int64_t layernorm_parts_most(int64_t cols) { return cols <= 2048 ? 592 : cols <= 4096 ? 296 : 148; }
// Rows that start anywhere need 8 | parts * (rows per block and turn), or a turn for all rows, so that all
// rows of a thread start alike: up to 8 parts.
inline int64_t layernorm_parts_bound(int64_t rows_per_group, int64_t groups, int64_t cols) {
  return std::min(rows_per_group, std::max<int64_t>(8, layernorm_parts_most(cols) / groups));
}
inline int64_t layernorm_parts(int64_t rows_per_group, int64_t groups, int64_t cols, int rows_per_turn, bool shift) {
  const int64_t turns = (rows_per_group + rows_per_turn - 1) / rows_per_turn;
  int64_t parts = std::max<int64_t>(1, layernorm_parts_most(cols) / groups);
  if (shift) {
    const int64_t unit = rows_per_turn >= 8 ? 1 : 8 / rows_per_turn;
    parts = std::max(unit, parts / unit * unit);
  }
  return std::min(parts, turns);
}

}  // namespace prm
