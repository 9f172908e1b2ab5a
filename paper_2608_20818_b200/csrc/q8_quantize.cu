// The quantiser: a matrix to 8-bit codes with one scale per row, per column, or both ways at once.
//
//   by rows:     t = x * fold_cols,   scale[i] = max_j |t_ij| / limit,   code = round(t * limit / max)
//   by columns:  t = x * fold_rows,   scale[j] = max_i |t_ij| / limit,   likewise
//
// The folds carry the scales that run along the sum of the product that will read the codes: a
// product can take out one factor per row of its left operand and per column of its right one, and
// nothing that varies inside its sums.
#include "q8.cuh"

namespace prm {
namespace {

struct QuantArgs {
  const void* x;
  const float* fold_rows;   // [rows] or null
  const float* fold_cols;   // [cols] or null
  uint8_t* q_rows;
  uint8_t* q_cols;
  float* scale_rows;
  float* scale_cols;
  uint32_t* top;            // [cols] largest magnitude of a column, as bits
  int64_t rows, ld_x, ld_qr, ld_qc;
  int cols, format;
};

template <int VEC>
__device__ __forceinline__ void fold_by_col(const float* f, int c, float (&t)[VEC]) {
  if (f) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = __fmul_rn(t[e], __ldg(f + c + e));
  }
}

// One row per group of TPR threads, in registers between the maximum and the rounding.
template <typename IO, int VEC, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) quantize_rows_kernel(const QuantArgs a) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  __shared__ uint32_t red[64];
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  float t[NV][VEC];
  float none = 0.f;
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + lane) * VEC;
    if (c < a.cols) {
      load_vec<VEC>(x + c, t[v]);
      fold_by_col<VEC>(a.fold_cols, c, t[v]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) top = max(top, abs_bits(t[v][e]));
    }
  }
  block_sum_max<TPR>(none, top, red);
  const Q8Scale s = q8_scale(top, q8_limit(a.format));
  uint8_t* q = a.q_rows + row * a.ld_qr;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + lane) * VEC;
    if (c < a.cols) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) t[v][e] = s.finite ? __fmul_rn(t[v][e], s.mul) : 0.f;
      store_codes<VEC>(q + c, t[v], a.format);
    }
  }
  if (lane == 0) a.scale_rows[row] = s.scale;
}

template <typename IO>
__global__ void __launch_bounds__(1024) quantize_rows_long_kernel(const QuantArgs a) {
  __shared__ uint32_t red[64];
  const int64_t row = blockIdx.x;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  float none = 0.f;
  uint32_t top = 0;
  for (int c = threadIdx.x; c < a.cols; c += 1024) {
    float t[1] = {to_f32(x[c])};
    fold_by_col<1>(a.fold_cols, c, t);
    top = max(top, abs_bits(t[0]));
  }
  block_sum_max<1024>(none, top, red);
  const Q8Scale s = q8_scale(top, q8_limit(a.format));
  for (int c = threadIdx.x; c < a.cols; c += 1024) {
    float t[1] = {to_f32(x[c])};
    fold_by_col<1>(a.fold_cols, c, t);
    a.q_rows[row * a.ld_qr + c] = q8_pack1(s.finite ? __fmul_rn(t[0], s.mul) : 0.f, a.format);
  }
  if (threadIdx.x == 0) a.scale_rows[row] = s.scale;
}

// Largest magnitude of every column: a block takes 256 * VEC columns of a slab of rows; the integer
// maximum joins the slabs in any order with the same result.
constexpr int kColThreads = 256;
template <typename IO, int VEC>
__global__ void __launch_bounds__(kColThreads) column_top_kernel(const QuantArgs a, int slab) {
  const int c = (blockIdx.x * kColThreads + threadIdx.x) * VEC;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * slab, r1 = min(a.rows, r0 + slab);
  uint32_t top[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) top[e] = 0;
  const IO* x = reinterpret_cast<const IO*>(a.x) + r0 * a.ld_x + c;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r, x += a.ld_x) {
    float t[VEC];
    load_vec<VEC>(x, t);
    const float f = a.fold_rows ? __ldg(a.fold_rows + r) : 1.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) top[e] = max(top[e], abs_bits(__fmul_rn(t[e], f)));
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) atomicMax(a.top + c + e, top[e]);
}

template <typename IO, int VEC>
__global__ void __launch_bounds__(kColThreads) quantize_cols_kernel(const QuantArgs a, int slab) {
  const int c = (blockIdx.x * kColThreads + threadIdx.x) * VEC;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * slab, r1 = min(a.rows, r0 + slab);
  Q8Scale s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = q8_scale(a.top[c + e], q8_limit(a.format));
  if (blockIdx.y == 0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) a.scale_cols[c + e] = s[e].scale;
  }
  const IO* x = reinterpret_cast<const IO*>(a.x) + r0 * a.ld_x + c;
  uint8_t* q = a.q_cols + r0 * a.ld_qc + c;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r, x += a.ld_x, q += a.ld_qc) {
    float t[VEC];
    load_vec<VEC>(x, t);
    const float f = a.fold_rows ? __ldg(a.fold_rows + r) : 1.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = s[e].finite ? __fmul_rn(__fmul_rn(t[e], f), s[e].mul) : 0.f;
    store_codes<VEC>(q, t, a.format);
  }
}

template <typename IO, int VEC, int NV, int TPR>
void launch_rows(const QuantArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  quantize_rows_kernel<IO, VEC, NV, TPR>
      <<<(unsigned)((a.rows + kRows - 1) / kRows), TPR == 32 ? 256 : TPR, 0, stream>>>(a);
}

template <typename IO>
void run_rows(const QuantArgs& a, bool vec, cudaStream_t stream) {
  const int c = a.cols;
  if (vec) {
    if (c <= 256) launch_rows<IO, 8, 1, 32>(a, stream);
    else if (c <= 512) launch_rows<IO, 8, 2, 32>(a, stream);
    else if (c <= 1024) launch_rows<IO, 8, 1, 128>(a, stream);
    else if (c <= 2048) launch_rows<IO, 8, 2, 128>(a, stream);
    else if (c <= 4096) launch_rows<IO, 8, 2, 256>(a, stream);
    else if (c <= 8192) launch_rows<IO, 8, 2, 512>(a, stream);
    else if (c <= 16384) launch_rows<IO, 8, 2, 1024>(a, stream);
    else if (c <= 32768) launch_rows<IO, 8, 4, 1024>(a, stream);
    else quantize_rows_long_kernel<IO><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
  } else {
    if (c <= 256) launch_rows<IO, 1, 8, 32>(a, stream);
    else if (c <= 2048) launch_rows<IO, 1, 8, 256>(a, stream);
    else if (c <= 8192) launch_rows<IO, 1, 16, 512>(a, stream);
    else if (c <= 16384) launch_rows<IO, 1, 16, 1024>(a, stream);
    else quantize_rows_long_kernel<IO><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
  }
}

template <typename IO, int VEC>
void run_cols(const QuantArgs& a, cudaStream_t stream) {
  const int bx = (a.cols + kColThreads * VEC - 1) / (kColThreads * VEC);
  // enough slabs for about eight blocks per SM, none shorter than 16 rows
  int64_t slabs = std::max<int64_t>(1, std::min<int64_t>((a.rows + 15) / 16, (8 * 148 + bx - 1) / bx));
  slabs = std::min<int64_t>(slabs, 65535);
  const int slab = (int)((a.rows + slabs - 1) / slabs);
  const dim3 grid((unsigned)bx, (unsigned)((a.rows + slab - 1) / slab));
  column_top_kernel<IO, VEC><<<grid, kColThreads, 0, stream>>>(a, slab);
  quantize_cols_kernel<IO, VEC><<<grid, kColThreads, 0, stream>>>(a, slab);
}

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" size_t prm_quantize_q8_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1) return 0;
  return (size_t)cols * 4;
}

extern "C" int prm_quantize_q8(const void* x, int64_t ld_x, int64_t rows, int64_t cols, int io_fp32, int format,
                               const float* fold_rows, const float* fold_cols, void* q_rows, int64_t ld_q_rows,
                               float* scale_rows, void* q_cols, int64_t ld_q_cols, float* scale_cols, void* scratch,
                               size_t scratch_bytes, void* cuda_stream) {
  if (!q8_format_ok(format) || rows < 0 || (!q_rows && !q_cols)) return PRM_ERR_ARG;
  if (cols < 1 || cols > 0x7fffffffLL - 8192 || rows > 0x7fffffffLL) return PRM_ERR_SHAPE;
  const int64_t most = (int64_t)1 << 40;
  if (ld_x < 0 || ld_x > most || (q_rows && (ld_q_rows < cols || ld_q_rows > most)) ||
      (q_cols && (ld_q_cols < cols || ld_q_cols > most)))
    return PRM_ERR_SHAPE;
  if ((q_rows && !scale_rows) || (q_cols && !scale_cols)) return PRM_ERR_ARG;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (((uintptr_t)scale_rows | (uintptr_t)scale_cols | (uintptr_t)fold_rows | (uintptr_t)fold_cols |
       (uintptr_t)scratch) % 4 != 0)
    return PRM_ERR_ALIGN;
  if (rows == 0) {                        // columns without an element: scale 0
    if (q_cols && cudaMemsetAsync(scale_cols, 0, (size_t)cols * 4, stream) != cudaSuccess) return PRM_ERR_CUDA;
    return PRM_OK;
  }
  if (!x) return PRM_ERR_ARG;
  if ((uintptr_t)x % (io_fp32 ? 4 : 2) != 0) return PRM_ERR_ALIGN;
  if (q_cols && (!scratch || scratch_bytes < prm_quantize_q8_scratch_bytes(rows, cols))) return PRM_ERR_WORKSPACE;
  QuantArgs a = {x, fold_rows, fold_cols, (uint8_t*)q_rows, (uint8_t*)q_cols, scale_rows, scale_cols,
                 (uint32_t*)scratch, rows, ld_x, ld_q_rows, ld_q_cols, (int)cols, format};
  const bool vec_x = cols % 8 == 0 && ld_x % 8 == 0 && aligned16(x);
  if (q_rows) {
    const bool vec = vec_x && ld_q_rows % 8 == 0 && ((uintptr_t)q_rows & 7) == 0;
    if (io_fp32) run_rows<float>(a, vec, stream);
    else run_rows<__nv_bfloat16>(a, vec, stream);
  }
  if (q_cols) {
    const bool vec = vec_x && ld_q_cols % 8 == 0 && ((uintptr_t)q_cols & 7) == 0;
    if (cudaMemsetAsync(scratch, 0, (size_t)cols * 4, stream) != cudaSuccess) return PRM_ERR_CUDA;
    if (io_fp32) {
      if (vec) run_cols<float, 8>(a, stream);
      else run_cols<float, 1>(a, stream);
    } else {
      if (vec) run_cols<__nv_bfloat16, 8>(a, stream);
      else run_cols<__nv_bfloat16, 1>(a, stream);
    }
  }
  return cudaGetLastError() == cudaSuccess ? PRM_OK : PRM_ERR_CUDA;
}
