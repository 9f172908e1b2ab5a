// Layer norm of a residual stream: dropout of the branch, the residual's addition, the norm, and a scale
// and shift that all rows or the rows of a group share.
//
//   h = [x dropped out] + r (stored in the stream's type),  mean = sum h / n,
//   rstd = 1 / sqrt(sum (h - mean)^2 / n + eps),            y = (h - mean) rstd w + b
//
// Bound by HBM (8 bytes per element of a bf16 stream with its residual): a row is read once and stays in
// registers, in octs (8 elements).  The squares are summed of h - mean, in a second reduction: from sums of h
// and h^2 a mean that is large against the deviations would cancel them.  That reduction sums h - mean too:
// what the first one's rounding has left in it (with a mean of 10^5 deviations, some 10^-2 of one) is taken off
// again from mean, variance and output.
#include "layernorm.cuh"

namespace prm {
namespace {

struct LayerNormArgs {
  const void* x;
  const void* residual;    // may be null
  void* h;                 // null: h = x, not stored
  void* y;
  float* mean;
  float* rstd;
  int64_t rows, ld_x, ld_r, ld_h, ld_y;
  int cols;
  uint32_t rows_per_group;
  float eps;
  Affine affine;
  Drop drop;
};

// Sums over a group of TPR threads (a block where TPR > 32); `red`: a word per warp, used once between two barriers.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = group_sum<(TPR < 32 ? TPR : 32)>(v);
  if constexpr (TPR > 32) {
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = threadIdx.x % 32 < TPR / 32 ? red[threadIdx.x % 32] : 0.f;
    v = warp_sum(v);
  }
  return v;
}
template <int TPR>
__device__ __forceinline__ float2 row_sum(float2 v, float2* red) {
  v.x = group_sum<(TPR < 32 ? TPR : 32)>(v.x);
  v.y = group_sum<(TPR < 32 ? TPR : 32)>(v.y);
  if constexpr (TPR > 32) {
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = threadIdx.x % 32 < TPR / 32 ? red[threadIdx.x % 32] : make_float2(0.f, 0.f);
    v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
  }
  return v;
}

// What the row's numbers are: mean and rstd, and what is still to be taken off h - (first mean).
struct RowStats {
  float mean, rstd, rest;
  // of the first mean, the sums of h - mean and of its squares
  __device__ __forceinline__ RowStats(float first, float2 sums, int cols, float eps) {
    rest = sums.x / (float)cols;
    mean = first + rest;
    rstd = 1.f / sqrtf(fmaxf(sums.y / (float)cols - rest * rest, 0.f) + eps);
  }
};

// One row per group of TPR threads (up to a warp: 256 / TPR rows per block; else a block), 8 * NV elements
// per thread.  SHIFT: octs aligned in memory, of rows that start anywhere.
template <typename IO, int NV, int TPR, bool DROP, bool SHIFT>
__global__ void __launch_bounds__(TPR <= 32 ? 256 : TPR) layernorm_kernel(const LayerNormArgs a) {
  constexpr int kRows = TPR <= 32 ? 256 / TPR : 1;
  __shared__ float red[32];
  __shared__ float2 red2[32];
  grid_wait();
  grid_trigger();
  const int64_t at = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  const int cols = at < a.rows ? a.cols : 0;                    // what this thread has of the row's columns
  const int64_t row = min(at, a.rows - 1), group = (uint32_t)row / a.rows_per_group;
  const OctRow<IO> x(a.x, row, a.rows, a.ld_x, a.cols);
  const OctRow<IO> r(a.residual ? a.residual : a.x, row, a.rows, a.residual ? a.ld_r : a.ld_x, a.cols);
  const int shift = SHIFT ? oct_shift(x.p) : 0;
  const int c0 = (int)(threadIdx.x % TPR) * 8 - shift;
  Oct<IO> xv[NV], rv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
      if constexpr (SHIFT) {
        x.load(c, cols, xv[v]);
        if (a.residual) r.load(c, cols, rv[v]);
      } else {
        xv[v].load_stream(x.p + c);
        if (a.residual) rv[v].load_stream(r.p + c);
      }
    }
  }
  const uint64_t number = DROP ? drop_number(a.drop) : 0;
  float2 t[NV][4], sum2 = make_float2(0.f, 0.f);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
      xv[v].get(t[v]);
      if constexpr (DROP) drop_oct<!SHIFT>(a.drop, number, (uint32_t)row, c, t[v]);
      if (a.residual) {
        float2 b[4];
        rv[v].get(b);
#pragma unroll
        for (int e = 0; e < 4; ++e) t[v][e] = add2(t[v][e], b[e]);
      }
      if (a.h) {
        IO* h = reinterpret_cast<IO*>(a.h) + row * a.ld_h;
        xv[v].set(t[v]);
        xv[v].get(t[v]);                                        // as it is stored
        if constexpr (SHIFT) store_part(h, c, cols, t[v]);
        else xv[v].store(h + c);
      }
      if constexpr (SHIFT) clear_outside(c, cols, t[v]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum2 = add2(sum2, t[v][e]);
    }
  }
  const float first = row_sum<TPR>(sum2.x + sum2.y, red) / (float)a.cols;
  float2 square2 = make_float2(0.f, 0.f);
  sum2 = square2;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
#pragma unroll
      for (int e = 0; e < 4; ++e) t[v][e] = add2(t[v][e], make_float2(-first, -first));
      if constexpr (SHIFT) clear_outside(c, cols, t[v]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum2 = add2(sum2, t[v][e]);
        square2 = fma2(t[v][e], t[v][e], square2);
      }
    }
  }
  const RowStats s(first, row_sum<TPR>(make_float2(sum2.x + sum2.y, square2.x + square2.y), red2), a.cols, a.eps);
  const float2 rs2 = make_float2(s.rstd, s.rstd), off2 = make_float2(-s.rest * s.rstd, -s.rest * s.rstd);
  IO* y = reinterpret_cast<IO*>(a.y) + row * a.ld_y;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
      float2 w[4], b[4];
      affine_weight(a.affine, group, c, cols, w);
      affine_bias(a.affine, group, c, cols, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[v][e] = fma2(fma2(t[v][e], rs2, off2), w[e], b[e]);
      if constexpr (SHIFT) {
        store_part(y, c, cols, t[v]);
      } else {
        xv[v].set(t[v]);
        xv[v].store(y + c);
      }
    }
  }
  if (threadIdx.x % TPR == 0 && cols) {
    a.mean[row] = s.mean;
    a.rstd[row] = s.rstd;
  }
}

// Any alignment, any length: three passes over the row, four elements per thread at a time, the later two of
// what the thread wrote itself (or of x).
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS) layernorm_single_kernel(const LayerNormArgs a) {
  __shared__ float red[32];
  __shared__ float2 red2[32];
  grid_wait();
  grid_trigger();
  const int64_t row = blockIdx.x, group = (uint32_t)row / a.rows_per_group;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  const IO* r = a.residual ? reinterpret_cast<const IO*>(a.residual) + row * a.ld_r : nullptr;
  IO* h = a.h ? reinterpret_cast<IO*>(a.h) + row * a.ld_h : nullptr;
  const uint64_t number = drop_number(a.drop);
  float sum = 0.f;
  for (int c = threadIdx.x * 4; c < a.cols; c += THREADS * 4) {
    uint4 w = make_uint4(~0u, ~0u, ~0u, ~0u);
    if (a.drop.threshold) w = drop_words(a.drop, number, (uint32_t)row, (uint32_t)c >> 2);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (c + k < a.cols) {
        float v = dropped(a.drop, word[k], to_f32(x[c + k]));
        if (r) v += to_f32(r[c + k]);
        if (h) {
          v = as_stored(v, (const IO*)nullptr);
          from_f32(h + c + k, v);
        }
        sum += v;
      }
    }
  }
  const float first = row_sum<THREADS>(sum, red) / (float)a.cols;
  const IO* src = h ? h : x;
  float2 sums = make_float2(0.f, 0.f);
  for (int c = threadIdx.x * 4; c < a.cols; c += THREADS * 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (c + k < a.cols) {
        const float v = to_f32(src[c + k]) - first;
        sums.x += v;
        sums.y += v * v;
      }
    }
  }
  const RowStats s(first, row_sum<THREADS>(sums, red2), a.cols, a.eps);
  IO* y = reinterpret_cast<IO*>(a.y) + row * a.ld_y;
  for (int c = threadIdx.x * 4; c < a.cols; c += THREADS * 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < a.cols)
        from_f32(y + c + k, (to_f32(src[c + k]) - first - s.rest) * s.rstd * affine_weight1(a.affine, group, c + k) +
                                affine_bias1(a.affine, group, c + k));
  }
  if (threadIdx.x == 0) {
    a.mean[row] = s.mean;
    a.rstd[row] = s.rstd;
  }
}

template <typename IO, bool DROP, bool SHIFT, int NV, int TPR>
int launch_layernorm(const LayerNormArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR <= 32 ? 256 / TPR : 1, kThreads = TPR <= 32 ? 256 : TPR;
  return q8_code(launch_after(layernorm_kernel<IO, NV, TPR, DROP, SHIFT>, (unsigned)((a.rows + kRows - 1) / kRows), kThreads,
                              0, stream, 0, a));
}

template <typename IO, bool DROP, bool SHIFT>
int run_layernorm(const LayerNormArgs& a, cudaStream_t stream) {
  const int64_t c = (int64_t)a.cols + (SHIFT ? 7 : 0);         // a row may need one more oct
  if (c <= 64) return launch_layernorm<IO, DROP, SHIFT, 1, 8>(a, stream);
  if (c <= 256) return launch_layernorm<IO, DROP, SHIFT, 1, 32>(a, stream);
  if (c <= 512) return launch_layernorm<IO, DROP, SHIFT, 2, 32>(a, stream);
  if (c <= 1024) return launch_layernorm<IO, DROP, SHIFT, 1, 128>(a, stream);
  if (c <= 2048) return launch_layernorm<IO, DROP, SHIFT, 2, 128>(a, stream);
  if (c <= 4096) return launch_layernorm<IO, DROP, SHIFT, 2, 256>(a, stream);
  if (c <= 8192) return launch_layernorm<IO, DROP, SHIFT, 2, 512>(a, stream);
  if (c <= 16384) return launch_layernorm<IO, DROP, SHIFT, 2, 1024>(a, stream);
  return q8_code(launch_after(layernorm_single_kernel<IO, 1024>, (unsigned)a.rows, 1024, 0, stream, 0, a));
}
template <typename IO>
int run_any(const LayerNormArgs& a, cudaStream_t stream) {
  const bool octs = a.cols % 8 == 0 && a.ld_x % 8 == 0 && a.ld_y % 8 == 0 && aligned16(a.x) && aligned16(a.y) &&
                    (!a.residual || (a.ld_r % 8 == 0 && aligned16(a.residual))) &&
                    (!a.h || (a.ld_h % 8 == 0 && aligned16(a.h)));
  const bool drop = a.drop.threshold != 0;
  if (octs) return drop ? run_layernorm<IO, true, false>(a, stream) : run_layernorm<IO, false, false>(a, stream);
  if (octs_alike<IO>(a.x, a.ld_x, a.y, a.ld_y) && (!a.residual || octs_alike<IO>(a.x, a.ld_x, a.residual, a.ld_r)) &&
      (!a.h || octs_alike<IO>(a.x, a.ld_x, a.h, a.ld_h)))
    return drop ? run_layernorm<IO, true, true>(a, stream) : run_layernorm<IO, false, true>(a, stream);
  if (a.cols <= 1024) return q8_code(launch_after(layernorm_single_kernel<IO, 128>, (unsigned)a.rows, 128, 0, stream, 0, a));
  return q8_code(launch_after(layernorm_single_kernel<IO, 1024>, (unsigned)a.rows, 1024, 0, stream, 0, a));
}

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" int prm_layernorm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight,
                             int64_t ld_weight, const void* bias, int64_t ld_bias, int64_t rows, int64_t cols,
                             int64_t rows_per_group, int io_fp32, int weight_fp32, int add_one, float eps, double p,
                             uint64_t seed, uint64_t offset, const uint64_t* counter, void* h_out, int64_t ld_h,
                             void* y_out, int64_t ld_y, float* mean_out, float* rstd_out, void* cuda_stream) {
  if (!(eps >= 0.f) || rows < 0 || rows_per_group < 1 || !drop_ok(p)) return PRM_ERR_ARG;
  if (cols < 1 || cols > 0x7fffffffLL - 8192 || rows > 0x7fffffffLL) return PRM_ERR_SHAPE;
  if (!layernorm_ld_ok(ld_x) || ld_y < cols || !layernorm_ld_ok(ld_y)) return PRM_ERR_SHAPE;
  if ((residual && !layernorm_ld_ok(ld_residual)) || (weight && !layernorm_ld_ok(ld_weight)) ||
      (bias && !layernorm_ld_ok(ld_bias)))
    return PRM_ERR_SHAPE;
  const Drop drop = make_drop(p, seed, offset, counter);
  const bool kept = residual || drop.threshold;
  if (kept && (ld_h < cols || !layernorm_ld_ok(ld_h))) return PRM_ERR_SHAPE;
  if (rows == 0) return PRM_OK;
  if (!x || !y_out || !mean_out || !rstd_out || (kept && !h_out)) return PRM_ERR_ARG;
  const uintptr_t stream_bits = (uintptr_t)x | (uintptr_t)residual | (uintptr_t)(kept ? h_out : nullptr) | (uintptr_t)y_out;
  if (stream_bits % (io_fp32 ? 4 : 2) != 0 || ((uintptr_t)weight | (uintptr_t)bias) % (weight_fp32 ? 4 : 2) != 0 ||
      ((uintptr_t)mean_out | (uintptr_t)rstd_out) % 4 != 0 || (uintptr_t)counter % 8 != 0)
    return PRM_ERR_ALIGN;
  const LayerNormArgs a = {x, residual, kept ? h_out : nullptr, y_out, mean_out, rstd_out, rows, ld_x, ld_residual, ld_h, ld_y,
                           (int)cols, (uint32_t)std::min<int64_t>(rows_per_group, rows), eps,
                           {weight, bias, ld_weight, ld_bias, weight_fp32, add_one}, drop};
  return io_fp32 ? run_any<float>(a, (cudaStream_t)cuda_stream) : run_any<__nv_bfloat16>(a, (cudaStream_t)cuda_stream);
}
