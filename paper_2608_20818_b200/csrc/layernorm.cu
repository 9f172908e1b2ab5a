// Layer norm of a residual stream: dropout of the branch, the residual's addition, the norm, and a scale
// and shift that all rows or the rows of a group share.
//
//   h = [x dropped out] + r (stored in the stream's type),  mean = sum h / n,
//   rstd = 1 / sqrt(sum (h - mean)^2 / n + eps),            y = (h - mean) rstd w + b
//
// Bound by HBM (8 bytes per element of a bf16 stream with its residual) and, close behind, by instructions: a row
// is read once and stays in registers, in octs (8 elements).  The squares are summed of h - mean, in a second reduction: from sums of h
// and h^2 a mean that is large against the deviations would cancel them.  That reduction sums h - mean too:
// what the first one's rounding has left in it (with a mean of 10^5 deviations, some 10^-2 of one) is taken off
// again from mean, variance and output.
//
// Measured: 8192 x 4096 in bf16 with residual 46 us, 5.8 TB/s (fp32 84 us, 6.4), with dropout 55 us; 16384 x 1024
// 27 us; 131072 x 128 24 us; 4096 x 16384 110 us, 4.9 TB/s (x 20480, by single elements, 283); one token of 2048 2 us.
// (Times here and below are the device's, of calls that follow one another on inputs beyond the L2.)
#include "layernorm_forward.cuh"

namespace prm {

int layernorm_aligned(const LayerNormArgs& a, const __nv_bfloat16*, cudaStream_t stream) {
  return a.drop.threshold ? run_layernorm<__nv_bfloat16, true, false>(a, stream) : run_layernorm<__nv_bfloat16, false, false>(a, stream);
}
int layernorm_aligned(const LayerNormArgs& a, const float*, cudaStream_t stream) {
  return a.drop.threshold ? run_layernorm<float, true, false>(a, stream) : run_layernorm<float, false, false>(a, stream);
}

namespace {

template <typename IO>
int run_any(const LayerNormArgs& a, cudaStream_t stream) {
  const bool octs = a.cols % 8 == 0 && a.ld_x % 8 == 0 && a.ld_y % 8 == 0 && aligned16(a.x) && aligned16(a.y) &&
                    (!a.residual || (a.ld_r % 8 == 0 && aligned16(a.residual))) &&
                    (!a.h || (a.ld_h % 8 == 0 && aligned16(a.h))) &&
                    (!a.affine.weight || (a.affine.ld_w % 8 == 0 && aligned16(a.affine.weight))) &&
                    (!a.affine.bias || (a.affine.ld_b % 8 == 0 && aligned16(a.affine.bias)));
  if (octs) return layernorm_aligned(a, (const IO*)nullptr, stream);
  if (octs_alike<IO>(a.x, a.ld_x, a.y, a.ld_y) && (!a.residual || octs_alike<IO>(a.x, a.ld_x, a.residual, a.ld_r)) &&
      (!a.h || octs_alike<IO>(a.x, a.ld_x, a.h, a.ld_h)))
    return layernorm_shifted(a, (const IO*)nullptr, stream);
  return run_layernorm_single<IO>(a, stream);
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
                           (int)cols, (uint32_t)std::min<int64_t>(rows_per_group, rows), 0, 0, eps, (float)(1.0 / (double)cols),
                           {weight, bias, ld_weight, ld_bias, weight_fp32, add_one}, drop};
  return io_fp32 ? run_any<float>(a, (cudaStream_t)cuda_stream) : run_any<__nv_bfloat16>(a, (cudaStream_t)cuda_stream);
}
