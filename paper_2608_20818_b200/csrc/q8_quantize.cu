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

// x * f for one oct (f: eight factors from c on, or null).
__device__ __forceinline__ void fold_oct(const float* f, int c, float2 (&t)[4]) {
  if (f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = mul2(t[e], make_float2(__ldg(f + c + 2 * e), __ldg(f + c + 2 * e + 1)));
  }
}

// One row per group of TPR threads, in registers between the maximum and the rounding.
template <typename IO, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) quantize_rows_kernel(const QuantArgs a) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  __shared__ float red[64];
  const int c0 = (threadIdx.x % TPR) * 8;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  Oct<IO> xv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (c0 + v * TPR * 8 < a.cols) xv[v].load_stream(x + c0 + v * TPR * 8);
  float2 t[NV][4];
  float none = 0.f, top = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < a.cols) {
      xv[v].get(t[v]);
      fold_oct(a.fold_cols, c, t[v]);
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max_abs(top, t[v][e]);
    }
  }
  block_sum_top<TPR>(none, top, red);
  const Q8Scale s = q8_scale(top, q8_limit(a.format));
  store_octs<NV>(a.q_rows + row * a.ld_qr, t, c0, TPR * 8, a.cols, s, a.format);
  if (c0 == 0) a.scale_rows[row] = s.scale;
}

// Any alignment, any length: two passes over the row.
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS) quantize_rows_single_kernel(const QuantArgs a) {
  __shared__ float red[64];
  const int64_t row = blockIdx.x;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  auto value = [&](int c) {
    const float v = to_f32(x[c]);
    return a.fold_cols ? __fmul_rn(v, __ldg(a.fold_cols + c)) : v;
  };
  float none = 0.f, top = 0.f;
#pragma unroll 4
  for (int c = threadIdx.x; c < a.cols; c += THREADS) top = max_abs(top, make_float2(value(c), 0.f));
  block_sum_top<THREADS>(none, top, red);
  const Q8Scale s = q8_scale(top, q8_limit(a.format));
#pragma unroll 4
  for (int c = threadIdx.x; c < a.cols; c += THREADS)
    a.q_rows[row * a.ld_qr + c] = code1(s.finite ? __fmul_rn(value(c), s.mul) : 0.f, a.format);
  if (threadIdx.x == 0) a.scale_rows[row] = s.scale;
}

// Largest magnitude of every column: a block takes 256 * VEC columns of a slab of rows; the maximum of
// the bit patterns (NaN above infinity above numbers) joins the slabs in any order alike.
constexpr int kColThreads = 256;
template <typename IO, int VEC>
__global__ void __launch_bounds__(kColThreads) column_top_kernel(const QuantArgs a, int slab) {
  const int c = (blockIdx.x * kColThreads + threadIdx.x) * VEC;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * slab, r1 = min(a.rows, r0 + slab);
  float top[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) top[e] = 0.f;
  const IO* x = reinterpret_cast<const IO*>(a.x) + r0 * a.ld_x + c;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r, x += a.ld_x) {
    const float f = a.fold_rows ? __ldg(a.fold_rows + r) : 1.f;
    if constexpr (VEC == 8) {
      Oct<IO> o;
      float2 t[4];
      o.load(x);
      o.get(t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        t[e] = mul2(t[e], make_float2(f, f));
        top[2 * e] = max_abs(top[2 * e], make_float2(t[e].x, 0.f));
        top[2 * e + 1] = max_abs(top[2 * e + 1], make_float2(t[e].y, 0.f));
      }
    } else {
      top[0] = max_abs(top[0], make_float2(__fmul_rn(to_f32(*x), f), 0.f));
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) atomicMax(a.top + c + e, __float_as_uint(top[e]));
}

template <typename IO, int VEC>
__global__ void __launch_bounds__(kColThreads) quantize_cols_kernel(const QuantArgs a, int slab) {
  const int c = (blockIdx.x * kColThreads + threadIdx.x) * VEC;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * slab, r1 = min(a.rows, r0 + slab);
  float mul[VEC];
  bool finite = true;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const Q8Scale s = q8_scale(__uint_as_float(a.top[c + e]), q8_limit(a.format));
    if (blockIdx.y == 0) a.scale_cols[c + e] = s.scale;
    mul[e] = s.mul;
    finite = finite && s.finite;
  }
  const IO* x = reinterpret_cast<const IO*>(a.x) + r0 * a.ld_x + c;
  uint8_t* q = a.q_cols + r0 * a.ld_qc + c;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r, x += a.ld_x, q += a.ld_qc) {
    const float f = a.fold_rows ? __ldg(a.fold_rows + r) : 1.f;
    float v[VEC];
    if constexpr (VEC == 8) {
      Oct<IO> o;
      float2 t[4];
      o.load(x);
      o.get(t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        t[e] = mul2(mul2(t[e], make_float2(f, f)), make_float2(mul[2 * e], mul[2 * e + 1]));
        v[2 * e] = t[e].x;
        v[2 * e + 1] = t[e].y;
      }
    } else {
      v[0] = __fmul_rn(__fmul_rn(to_f32(*x), f), mul[0]);
    }
    if (!finite) {                        // a column without a scale: its codes are zero
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = a.top[c + e] < 0x7f800000u ? v[e] : 0.f;
    }
    if constexpr (VEC == 8) {
      const float2 p0 = make_float2(v[0], v[1]), p1 = make_float2(v[2], v[3]), p2 = make_float2(v[4], v[5]),
                   p3 = make_float2(v[6], v[7]);
      *reinterpret_cast<uint2*>(q) =
          a.format == PRM_Q8_INT8 ? make_uint2(codes4<PRM_Q8_INT8>(p0, p1), codes4<PRM_Q8_INT8>(p2, p3))
                                  : make_uint2(codes4<PRM_Q8_E4M3>(p0, p1), codes4<PRM_Q8_E4M3>(p2, p3));
    } else {
      *q = code1(v[0], a.format);
    }
  }
}

template <typename IO, int NV, int TPR>
void launch_rows(const QuantArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  quantize_rows_kernel<IO, NV, TPR>
      <<<(unsigned)((a.rows + kRows - 1) / kRows), TPR == 32 ? 256 : TPR, 0, stream>>>(a);
}

template <typename IO>
void run_rows(const QuantArgs& a, bool octs, cudaStream_t stream) {
  const int c = a.cols;
  if (octs && c <= 16384) {
    if (c <= 256) launch_rows<IO, 1, 32>(a, stream);
    else if (c <= 512) launch_rows<IO, 2, 32>(a, stream);
    else if (c <= 1024) launch_rows<IO, 1, 128>(a, stream);
    else if (c <= 2048) launch_rows<IO, 2, 128>(a, stream);
    else if (c <= 4096) launch_rows<IO, 2, 256>(a, stream);
    else if (c <= 8192) launch_rows<IO, 2, 512>(a, stream);
    else launch_rows<IO, 2, 1024>(a, stream);
  } else {
    if (c <= 1024) quantize_rows_single_kernel<IO, 128><<<(unsigned)a.rows, 128, 0, stream>>>(a);
    else if (c <= 8192) quantize_rows_single_kernel<IO, 256><<<(unsigned)a.rows, 256, 0, stream>>>(a);
    else quantize_rows_single_kernel<IO, 1024><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
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
