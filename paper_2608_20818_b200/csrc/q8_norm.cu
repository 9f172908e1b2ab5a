// Root-mean-square norm with the residual's addition and an 8-bit output, and its gradient.
//
//   h = x + r (stored in the stream's type),  t = h * w,  T = max |t| over the row
//   code = round(t * limit / T),   scale = T / limit * s,   s = 1 / sqrt(mean h^2 + eps)
//
// The norm's output is t * s; s is common to the row, so it cancels from the codes and one
// reduction gives the two numbers a row needs (T and the sum of squares).
//
// Gradient, the rounding taken as the identity, with g = grad_y * w:
//   grad_x = s g - h s^3 mean(g h) + grad_h,    grad_w = sum over rows of grad_y h s
#include "q8.cuh"

namespace prm {
namespace {

struct NormArgs {
  const void* x;
  const void* residual;   // may be null
  const void* weight;
  void* h;                // may be null without a residual
  uint8_t* q;
  float* scale;
  int64_t rows, ld_x, ld_r, ld_h, ld_q;
  int cols, weight_fp32, format;
  float eps;
};

// One row per group of TPR threads (a warp: eight rows per block; else a block), kept in registers
// between the reduction and the rounding: VEC * NV elements per thread.
template <typename IO, int VEC, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) rmsnorm_q8_kernel(const NormArgs a) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  __shared__ uint32_t red[64];
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;              // whole warps (kRows > 1) or no thread
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  const IO* r = a.residual ? reinterpret_cast<const IO*>(a.residual) + row * a.ld_r : nullptr;
  float t[NV][VEC];
  float sum = 0.f;
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + lane) * VEC;
    if (c < a.cols) {
      load_vec<VEC>(x + c, t[v]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) t[v][e] = 0.f;
    }
  }
  if (r) {
    IO* h = reinterpret_cast<IO*>(a.h) + row * a.ld_h;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + lane) * VEC;
      if (c < a.cols) {
        float b[VEC];
        load_vec<VEC>(r + c, b);
#pragma unroll
        for (int e = 0; e < VEC; ++e) t[v][e] = as_stored(t[v][e] + b[e], (const IO*)nullptr);
        store_vec<VEC>(h + c, t[v]);
      }
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + lane) * VEC;
    if (c < a.cols) {
      float w[VEC];
      load_weight<VEC>(a.weight, a.weight_fp32, c, w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        sum += t[v][e] * t[v][e];
        t[v][e] = __fmul_rn(t[v][e], w[e]);
        top = max(top, abs_bits(t[v][e]));
      }
    }
  }
  block_sum_max<TPR>(sum, top, red);
  const Q8Scale s = q8_scale(top, q8_limit(a.format));
  uint8_t* q = a.q + row * a.ld_q;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + lane) * VEC;
    if (c < a.cols) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) t[v][e] = s.finite ? __fmul_rn(t[v][e], s.mul) : 0.f;
      store_codes<VEC>(q + c, t[v], a.format);
    }
  }
  if (lane == 0) a.scale[row] = s.scale * (1.f / sqrtf(sum / (float)a.cols + a.eps));
}

// Rows too long for the registers of a block: the same in two passes over the row, the second of
// which finds it in L2.
template <typename IO>
__global__ void __launch_bounds__(1024) rmsnorm_q8_long_kernel(const NormArgs a) {
  __shared__ uint32_t red[64];
  const int64_t row = blockIdx.x;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  const IO* r = a.residual ? reinterpret_cast<const IO*>(a.residual) + row * a.ld_r : nullptr;
  IO* h = r ? reinterpret_cast<IO*>(a.h) + row * a.ld_h : nullptr;
  float sum = 0.f;
  uint32_t top = 0;
  for (int c = threadIdx.x; c < a.cols; c += 1024) {
    float v = to_f32(x[c]);
    if (r) {
      v = as_stored(v + to_f32(r[c]), (const IO*)nullptr);
      from_f32(h + c, v);
    }
    float w[1];
    load_weight<1>(a.weight, a.weight_fp32, c, w);
    sum += v * v;
    top = max(top, abs_bits(__fmul_rn(v, w[0])));
  }
  block_sum_max<1024>(sum, top, red);
  const Q8Scale s = q8_scale(top, q8_limit(a.format));
  const IO* src = r ? h : x;
  uint8_t* q = a.q + row * a.ld_q;
  for (int c = threadIdx.x; c < a.cols; c += 1024) {      // each thread reads what it wrote itself
    float w[1];
    load_weight<1>(a.weight, a.weight_fp32, c, w);
    const float t = __fmul_rn(to_f32(src[c]), w[0]);
    q[c] = q8_pack1(s.finite ? __fmul_rn(t, s.mul) : 0.f, a.format);
  }
  if (threadIdx.x == 0) a.scale[row] = s.scale * (1.f / sqrtf(sum / (float)a.cols + a.eps));
}

template <typename IO, int VEC, int NV, int TPR>
void launch_norm(const NormArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  rmsnorm_q8_kernel<IO, VEC, NV, TPR>
      <<<(unsigned)((a.rows + kRows - 1) / kRows), TPR == 32 ? 256 : TPR, 0, stream>>>(a);
}

template <typename IO>
void run_norm(const NormArgs& a, bool vec, cudaStream_t stream) {
  const int c = a.cols;
  if (vec) {
    if (c <= 256) launch_norm<IO, 8, 1, 32>(a, stream);
    else if (c <= 512) launch_norm<IO, 8, 2, 32>(a, stream);
    else if (c <= 1024) launch_norm<IO, 8, 1, 128>(a, stream);
    else if (c <= 2048) launch_norm<IO, 8, 2, 128>(a, stream);
    else if (c <= 4096) launch_norm<IO, 8, 2, 256>(a, stream);
    else if (c <= 8192) launch_norm<IO, 8, 2, 512>(a, stream);
    else if (c <= 16384) launch_norm<IO, 8, 2, 1024>(a, stream);
    else if (c <= 32768) launch_norm<IO, 8, 4, 1024>(a, stream);
    else rmsnorm_q8_long_kernel<IO><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
  } else {
    if (c <= 256) launch_norm<IO, 1, 8, 32>(a, stream);
    else if (c <= 2048) launch_norm<IO, 1, 8, 256>(a, stream);
    else if (c <= 8192) launch_norm<IO, 1, 16, 512>(a, stream);
    else if (c <= 16384) launch_norm<IO, 1, 16, 1024>(a, stream);
    else rmsnorm_q8_long_kernel<IO><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
  }
}

// ------------------------------------------------------------------ gradient

struct NormGradArgs {
  const void* gy;
  const void* h;
  const void* weight;
  const void* gh;         // may be null
  void* gx;
  float* part;            // [parts][cols] partial sums of grad_w
  int64_t rows, ld_gy, ld_h, ld_gh, ld_gx;
  int cols, weight_fp32;
  float eps;
};

// Sums of two numbers over a block.
template <int THREADS>
__device__ __forceinline__ void block_sum2(float& p, float& q, float* red) {
  p = warp_sum(p);
  q = warp_sum(q);
  if constexpr (THREADS > 32) {
    constexpr int kWarps = THREADS / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
      red[warp] = p;
      red[32 + warp] = q;
    }
    __syncthreads();
    p = lane < kWarps ? red[lane] : 0.f;
    q = lane < kWarps ? red[32 + lane] : 0.f;
    p = warp_sum(p);
    q = warp_sum(q);
  }
}

// A block walks over rows; a thread keeps the same columns in all of them, so its share of grad_w
// stays in registers until the block's last row.
template <typename IO, int VEC, int NV, int TPR>
__global__ void __launch_bounds__(TPR) rmsnorm_q8_grad_kernel(const NormGradArgs a) {
  __shared__ float red[2][64];
  const int lane = threadIdx.x;
  float gw[NV][VEC];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < VEC; ++e) gw[v][e] = 0.f;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const IO* gyp = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
    const IO* hp = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
    float gy[NV][VEC], h[NV][VEC];
    float ss = 0.f, gh = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + lane) * VEC;
      if (c < a.cols) {
        float w[VEC];
        load_vec<VEC>(gyp + c, gy[v]);
        load_vec<VEC>(hp + c, h[v]);
        load_weight<VEC>(a.weight, a.weight_fp32, c, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          ss += h[v][e] * h[v][e];
          gh += gy[v][e] * w[e] * h[v][e];
        }
      }
    }
    block_sum2<TPR>(ss, gh, red[turn]);
    const float s = 1.f / sqrtf(ss / (float)a.cols + a.eps);
    const float k = s * s * s * (gh / (float)a.cols);
    const IO* ghp = a.gh ? reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh : nullptr;
    IO* gxp = reinterpret_cast<IO*>(a.gx) + row * a.ld_gx;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + lane) * VEC;
      if (c < a.cols) {
        float w[VEC], out[VEC];
        load_weight<VEC>(a.weight, a.weight_fp32, c, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          gw[v][e] += gy[v][e] * h[v][e] * s;
          out[e] = s * (gy[v][e] * w[e]) - h[v][e] * k;
        }
        if (ghp) {
          float d[VEC];
          load_vec<VEC>(ghp + c, d);
#pragma unroll
          for (int e = 0; e < VEC; ++e) out[e] += d[e];
        }
        store_vec<VEC>(gxp + c, out);
      }
    }
  }
  float* part = a.part + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + lane) * VEC;
    if (c < a.cols) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) part[c + e] = gw[v][e];
    }
  }
}

// Rows too long for registers: two passes over the row, and the block's share of grad_w collected
// in its line of the scratch (each thread its own columns).
template <typename IO>
__global__ void __launch_bounds__(1024) rmsnorm_q8_grad_long_kernel(const NormGradArgs a) {
  __shared__ float red[2][64];
  float* part = a.part + (int64_t)blockIdx.x * a.cols;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const IO* gyp = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
    const IO* hp = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
    const IO* ghp = a.gh ? reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh : nullptr;
    IO* gxp = reinterpret_cast<IO*>(a.gx) + row * a.ld_gx;
    float ss = 0.f, gh = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      float w[1];
      load_weight<1>(a.weight, a.weight_fp32, c, w);
      const float h = to_f32(hp[c]);
      ss += h * h;
      gh += to_f32(gyp[c]) * w[0] * h;
    }
    block_sum2<1024>(ss, gh, red[turn]);
    const float s = 1.f / sqrtf(ss / (float)a.cols + a.eps);
    const float k = s * s * s * (gh / (float)a.cols);
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
      float w[1];
      load_weight<1>(a.weight, a.weight_fp32, c, w);
      const float h = to_f32(hp[c]), gy = to_f32(gyp[c]);
      float out = s * (gy * w[0]) - h * k;
      if (ghp) out += to_f32(ghp[c]);
      from_f32(gxp + c, out);
      const float add = gy * h * s;
      part[c] = row == (int64_t)blockIdx.x ? add : part[c] + add;
    }
  }
}

// grad_w: the parts added in a fixed order, 32 columns per block, eight parts at a time.
__global__ void __launch_bounds__(256)
rmsnorm_q8_grad_weight_kernel(const float* part, int parts, int cols, void* gw, int fp32) {
  __shared__ float s[8][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), k = threadIdx.x >> 5;
  float sum = 0.f;
  if (c < cols)
    for (int p = k; p < parts; p += 8) sum += part[(int64_t)p * cols + c];
  s[k][threadIdx.x & 31] = sum;
  __syncthreads();
  if (k == 0 && c < cols) {
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += s[j][threadIdx.x];
    if (fp32) reinterpret_cast<float*>(gw)[c] = sum;
    else reinterpret_cast<__nv_bfloat16*>(gw)[c] = __float2bfloat16_rn(sum);
  }
}

constexpr int kGradParts = 296;    // two blocks per SM

int grad_parts(int64_t rows) { return (int)std::min<int64_t>(rows, kGradParts); }

template <typename IO, int VEC, int NV, int TPR>
void launch_grad(const NormGradArgs& a, int parts, cudaStream_t stream) {
  rmsnorm_q8_grad_kernel<IO, VEC, NV, TPR><<<parts, TPR, 0, stream>>>(a);
}

template <typename IO>
void run_grad(const NormGradArgs& a, bool vec, int parts, cudaStream_t stream) {
  const int c = a.cols;
  if (vec) {
    if (c <= 256) launch_grad<IO, 8, 1, 32>(a, parts, stream);
    else if (c <= 1024) launch_grad<IO, 8, 1, 128>(a, parts, stream);
    else if (c <= 2048) launch_grad<IO, 8, 1, 256>(a, parts, stream);
    else if (c <= 4096) launch_grad<IO, 8, 1, 512>(a, parts, stream);
    else if (c <= 8192) launch_grad<IO, 8, 1, 1024>(a, parts, stream);
    else rmsnorm_q8_grad_long_kernel<IO><<<parts, 1024, 0, stream>>>(a);
  } else {
    if (c <= 256) launch_grad<IO, 1, 8, 32>(a, parts, stream);
    else if (c <= 2048) launch_grad<IO, 1, 8, 256>(a, parts, stream);
    else if (c <= 8192) launch_grad<IO, 1, 8, 1024>(a, parts, stream);
    else rmsnorm_q8_grad_long_kernel<IO><<<parts, 1024, 0, stream>>>(a);
  }
}

bool ld_ok(int64_t ld) { return ld >= 0 && ld <= ((int64_t)1 << 40); }

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" int prm_rmsnorm_q8(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual,
                              const void* weight, int64_t rows, int64_t cols, int io_fp32, int weight_fp32,
                              float eps, int format, void* h_out, int64_t ld_h, void* q_out, int64_t ld_q,
                              float* scale_out, void* cuda_stream) {
  if (!q8_format_ok(format) || !(eps >= 0.f) || rows < 0) return PRM_ERR_ARG;
  if (cols < 1 || cols > 0x7fffffffLL - 8192 || rows > 0x7fffffffLL) return PRM_ERR_SHAPE;
  if (!ld_ok(ld_x) || ld_q < cols || !ld_ok(ld_q)) return PRM_ERR_SHAPE;
  if (residual && (!ld_ok(ld_residual) || ld_h < cols || !ld_ok(ld_h))) return PRM_ERR_SHAPE;
  if (rows == 0) return PRM_OK;
  if (!x || !weight || !q_out || !scale_out || (residual && !h_out)) return PRM_ERR_ARG;
  const int es = io_fp32 ? 4 : 2;
  if (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)(residual ? h_out : nullptr)) % es != 0 ||
      (uintptr_t)weight % (weight_fp32 ? 4 : 2) != 0 || (uintptr_t)scale_out % 4 != 0)
    return PRM_ERR_ALIGN;
  NormArgs a = {x, residual, weight, h_out, (uint8_t*)q_out, scale_out, rows, ld_x, ld_residual, ld_h, ld_q,
                (int)cols, weight_fp32, format, eps};
  const bool vec = cols % 8 == 0 && ld_x % 8 == 0 && ld_q % 8 == 0 && aligned16(x) && aligned16(weight) &&
                   ((uintptr_t)q_out & 7) == 0 &&
                   (!residual || (ld_residual % 8 == 0 && ld_h % 8 == 0 && aligned16(residual) && aligned16(h_out)));
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (io_fp32) run_norm<float>(a, vec, stream);
  else run_norm<__nv_bfloat16>(a, vec, stream);
  return cudaGetLastError() == cudaSuccess ? PRM_OK : PRM_ERR_CUDA;
}

extern "C" size_t prm_rmsnorm_q8_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1) return 0;
  return (size_t)grad_parts(rows) * (size_t)cols * 4;
}

extern "C" int prm_rmsnorm_q8_backward(const void* grad_y, int64_t ld_grad_y, const void* h, int64_t ld_h,
                                       const void* weight, const void* grad_h, int64_t ld_grad_h, int64_t rows,
                                       int64_t cols, int io_fp32, int weight_fp32, float eps, void* grad_x,
                                       int64_t ld_grad_x, void* grad_weight, void* scratch, size_t scratch_bytes,
                                       void* cuda_stream) {
  if (!(eps >= 0.f) || rows < 0) return PRM_ERR_ARG;
  if (cols < 1 || cols > 0x7fffffffLL - 8192 || rows > 0x7fffffffLL) return PRM_ERR_SHAPE;
  if (!ld_ok(ld_grad_y) || !ld_ok(ld_h) || (grad_h && !ld_ok(ld_grad_h)) || ld_grad_x < cols || !ld_ok(ld_grad_x))
    return PRM_ERR_SHAPE;
  if (!grad_weight) return PRM_ERR_ARG;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if ((uintptr_t)grad_weight % (weight_fp32 ? 4 : 2) != 0) return PRM_ERR_ALIGN;
  if (rows == 0)                          // an empty sum
    return cudaMemsetAsync(grad_weight, 0, (size_t)cols * (weight_fp32 ? 4 : 2), stream) == cudaSuccess ? PRM_OK
                                                                                                     : PRM_ERR_CUDA;
  if (!grad_y || !h || !weight || !grad_x || !scratch) return PRM_ERR_ARG;
  if (scratch_bytes < prm_rmsnorm_q8_scratch_bytes(rows, cols)) return PRM_ERR_WORKSPACE;
  const int es = io_fp32 ? 4 : 2;
  if (((uintptr_t)grad_y | (uintptr_t)h | (uintptr_t)grad_h | (uintptr_t)grad_x) % es != 0 ||
      (uintptr_t)weight % (weight_fp32 ? 4 : 2) != 0 || ((uintptr_t)scratch & 15) != 0)
    return PRM_ERR_ALIGN;
  NormGradArgs a = {grad_y, h, weight, grad_h, grad_x, (float*)scratch, rows, ld_grad_y, ld_h, ld_grad_h, ld_grad_x,
                    (int)cols, weight_fp32, eps};
  const bool vec = cols % 8 == 0 && ld_grad_y % 8 == 0 && ld_h % 8 == 0 && ld_grad_x % 8 == 0 && aligned16(grad_y) &&
                   aligned16(h) && aligned16(grad_x) && aligned16(weight) &&
                   (!grad_h || (ld_grad_h % 8 == 0 && aligned16(grad_h)));
  const int parts = grad_parts(rows);
  if (io_fp32) run_grad<float>(a, vec, parts, stream);
  else run_grad<__nv_bfloat16>(a, vec, parts, stream);
  rmsnorm_q8_grad_weight_kernel<<<(unsigned)((cols + 31) / 32), 256, 0, stream>>>(a.part, parts, (int)cols,
                                                                                grad_weight, weight_fp32);
  return cudaGetLastError() == cudaSuccess ? PRM_OK : PRM_ERR_CUDA;
}
