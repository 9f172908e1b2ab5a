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
//
// Both are bound by HBM (7 and 8 bytes per element of a bf16 stream with its residual), so a row is read
// once and stays in registers, in octs (8 elements), between its sums and its output.  Measured on 8192
// x 4096 in bf16 with residual: norm 38.2 us, 6.1 TB/s; gradient 52.3 us, 5.1 TB/s (it also waits for
// the whole grid to add grad_w).  For one token each takes 2 to 5 us, the launch and one trip to memory.
// (Times here and below are the device's, of calls that follow one another on inputs beyond the L2.)
// Forms: rows of aligned octs; octs aligned in memory for rows that start anywhere; the gradient of rows
// of 4097 to 8192 streamed through shared memory; and single elements in two passes for what is left.
#include <cooperative_groups.h>

#include "row_ring.cuh"

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
  float minus_zero = -0.f;   // see int8_bits
};

__device__ __forceinline__ float inv_rms(float sum, int cols, float eps) { return 1.f / sqrtf(sum / (float)cols + eps); }

// A row that counts as zero has the scale 0 with eps = 0 too.
__device__ __forceinline__ float norm_scale(float top, float sum, const NormArgs& a) {
  const float u = q8_scale(top, q8_limit(a.format));
  return u == 0.f ? 0.f : u * inv_rms(sum, a.cols, a.eps);
}

template <typename T>
__device__ __forceinline__ void load_oct(const T* p, float2 (&v)[4]) {
  Oct<T> o;
  o.load(p);
  o.get(v);
}
// h (= x, plus r if RES, rounded to the stream's type and stored), t = h * w, sum of squares and top.
template <typename IO, bool RES>
__device__ __forceinline__ void norm_oct(Oct<IO> x, Oct<IO> r, const float2 (&w)[4], IO* h_out, float2 (&t)[4],
                                         float2& sum, float& top) {
  if constexpr (RES) {
    float2 b[4];
    x.get(t);
    r.get(b);
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = add2(t[e], b[e]);
    x.set(t);
    x.store(h_out);
  }
  x.get(t);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sum = fma2(t[e], t[e], sum);
    t[e] = mul2(t[e], w[e]);
    top = max_abs(top, t[e]);
  }
}

// One row per group of TPR threads (up to a warp: 256 / TPR rows per block; else a block), 8 * NV elements
// per thread.
template <typename IO, typename WT, int NV, int TPR, bool RES>
__global__ void __launch_bounds__(TPR <= 32 ? 256 : TPR) rmsnorm_q8_kernel(const NormArgs a) {
  constexpr int kRows = TPR <= 32 ? 256 / TPR : 1;
  __shared__ float red[64];
  grid_wait();
  grid_trigger();
  const int c0 = (threadIdx.x % TPR) * 8;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  const int cols = row < a.rows ? a.cols : 0;                   // what this thread has of the row's columns
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  const IO* r = RES ? reinterpret_cast<const IO*>(a.residual) + row * a.ld_r : nullptr;
  IO* h = RES ? reinterpret_cast<IO*>(a.h) + row * a.ld_h : nullptr;
  Oct<IO> xv[NV], rv[NV];
  Oct<WT> wv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
      xv[v].load_stream(x + c);
      if constexpr (RES) rv[v].load_stream(r + c);
      else rv[v].zero();
      wv[v].load(reinterpret_cast<const WT*>(a.weight) + c);
    }
  }
  float2 t[NV][4], sum2 = make_float2(0.f, 0.f);
  float top = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
      float2 w[4];
      wv[v].get(w);
      norm_oct<IO, RES>(xv[v], rv[v], w, h + c, t[v], sum2, top);
    }
  }
  float sum = sum2.x + sum2.y;
  block_sum_top<TPR>(sum, top, red);
  store_octs<NV>(a.q + row * a.ld_q, t, c0, TPR * 8, cols, top, a.format, a.minus_zero);
  if (c0 == 0 && cols) a.scale[row] = norm_scale(top, sum, a);
}

// Rows that start anywhere (odd widths), or too wide for the kernels above: as rmsnorm_q8_kernel, on
// octs aligned in memory.
template <typename IO, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) rmsnorm_q8_shifted_kernel(const NormArgs a) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  __shared__ float red[64];
  __shared__ uint64_t stage[kRows][NV * TPR + 1];
  grid_wait();
  grid_trigger();
  const int o0 = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;
  const OctRow<IO> x(a.x, row, a.rows, a.ld_x, a.cols);
  const OctRow<IO> r(a.residual ? a.residual : a.x, row, a.rows, a.residual ? a.ld_r : a.ld_x, a.cols);
  const int shift = oct_shift(x.p);
  Oct<IO> xv[NV], rv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (o0 + v * TPR) * 8 - shift;
    x.load(c, a.cols, xv[v]);
    if (a.residual) r.load(c, a.cols, rv[v]);
  }
  float2 t[NV][4], sum2 = make_float2(0.f, 0.f);
  float top = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (o0 + v * TPR) * 8 - shift;
    float2 w[4];
    load_factors(a.weight, a.weight_fp32, c, a.cols, w);
    get_part(xv[v], c, a.cols, t[v]);
    if (a.residual) {
      float2 b[4];
      get_part(rv[v], c, a.cols, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[v][e] = add2(t[v][e], b[e]);
      xv[v].set(t[v]);
      xv[v].get(t[v]);
      store_part(reinterpret_cast<IO*>(a.h) + row * a.ld_h, c, a.cols, t[v]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum2 = fma2(t[v][e], t[v][e], sum2);
      t[v][e] = mul2(t[v][e], w[e]);
      top = max_abs(top, t[v][e]);
    }
  }
  float sum = sum2.x + sum2.y;
  block_sum_top<TPR>(sum, top, red);
  store_octs_shifted<NV, TPR>(stage[threadIdx.x / TPR], a.q + row * a.ld_q, t, o0, shift, a.cols, top, a.format, a.minus_zero);
  if (o0 == 0) a.scale[row] = norm_scale(top, sum, a);
}

// Any alignment, any length: two passes over the row, the second of which finds it in cache.
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS) rmsnorm_q8_single_kernel(const NormArgs a) {
  __shared__ float red[64];
  grid_wait();
  grid_trigger();
  const int64_t row = blockIdx.x;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  const IO* r = a.residual ? reinterpret_cast<const IO*>(a.residual) + row * a.ld_r : nullptr;
  IO* h = r ? reinterpret_cast<IO*>(a.h) + row * a.ld_h : nullptr;
  float sum = 0.f, top = 0.f;
#pragma unroll 4
  for (int c = threadIdx.x; c < a.cols; c += THREADS) {
    float v = to_f32(x[c]);
    if (r) {
      v = as_stored(v + to_f32(r[c]), (const IO*)nullptr);
      from_f32(h + c, v);
    }
    sum += v * v;
    top = max_abs(top, make_float2(__fmul_rn(v, load1(a.weight, a.weight_fp32, c)), 0.f));
  }
  block_sum_top<THREADS>(sum, top, red);
  const bool finite = q8_finite(top);
  const float mul = q8_mul(top, q8_limit(a.format));
  const IO* src = r ? h : x;
  uint8_t* q = a.q + row * a.ld_q;
#pragma unroll 4
  for (int c = threadIdx.x; c < a.cols; c += THREADS) {      // each thread reads what it wrote itself
    const float t = __fmul_rn(to_f32(src[c]), load1(a.weight, a.weight_fp32, c));
    q[c] = finite ? code1(t, mul, a.format) : 0;
  }
  if (threadIdx.x == 0) a.scale[row] = norm_scale(top, sum, a);
}

template <typename IO, typename WT, int NV, int TPR>
int launch_norm(const NormArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR <= 32 ? 256 / TPR : 1, kThreads = TPR <= 32 ? 256 : TPR;
  const unsigned blocks = (unsigned)((a.rows + kRows - 1) / kRows);
  return q8_code(launch_after(a.residual ? rmsnorm_q8_kernel<IO, WT, NV, TPR, true> : rmsnorm_q8_kernel<IO, WT, NV, TPR, false>,
                              blocks, kThreads, 0, stream, 0, a));
}

template <typename IO, typename WT>
int run_norm(const NormArgs& a, cudaStream_t stream) {
  const int c = a.cols;
  if (c <= 64) return launch_norm<IO, WT, 1, 8>(a, stream);
  if (c <= 128) return launch_norm<IO, WT, 1, 16>(a, stream);
  if (c <= 256) return launch_norm<IO, WT, 1, 32>(a, stream);
  if (c <= 512) return launch_norm<IO, WT, 2, 32>(a, stream);
  // One block per row costs 1 ns each, more than a short row's bytes (16384 x 1024 without residual: 18.2 us,
  // eight rows per block 14.3); few rows end sooner with more threads (256 x 1024: 2.2 us, a warp 2.6).
  if (c <= 1024 && a.rows >= 2048) return launch_norm<IO, WT, 4, 32>(a, stream);
  if (c <= 1024) return launch_norm<IO, WT, 1, 128>(a, stream);
  if (c <= 2048) return launch_norm<IO, WT, 2, 128>(a, stream);
  if (c <= 4096) return launch_norm<IO, WT, 2, 256>(a, stream);
  if (c <= 8192) return launch_norm<IO, WT, 2, 512>(a, stream);
  return launch_norm<IO, WT, 2, 1024>(a, stream);
}

template <typename IO, int NV, int TPR>
int launch_norm_shifted(const NormArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  return q8_code(launch_after(rmsnorm_q8_shifted_kernel<IO, NV, TPR>, (unsigned)((a.rows + kRows - 1) / kRows),
                              TPR == 32 ? 256 : TPR, 0, stream, 0, a));
}

// `alike`: the matrices' rows start alike and the codes' rows on 8 bytes.
template <typename IO>
int run_norm_single(const NormArgs& a, bool alike, cudaStream_t stream) {
  const int c = a.cols + 7;               // a row may need one more oct
  if (alike && c <= 32768) {
    if (c <= 256) return launch_norm_shifted<IO, 1, 32>(a, stream);
    if (c <= 512) return launch_norm_shifted<IO, 2, 32>(a, stream);
    if (c <= 1024) return launch_norm_shifted<IO, 1, 128>(a, stream);
    if (c <= 2048) return launch_norm_shifted<IO, 2, 128>(a, stream);
    if (c <= 3072) return launch_norm_shifted<IO, 3, 128>(a, stream);
    if (c <= 4096) return launch_norm_shifted<IO, 2, 256>(a, stream);
    if (c <= 6144) return launch_norm_shifted<IO, 3, 256>(a, stream);
    if (c <= 8192) return launch_norm_shifted<IO, 2, 512>(a, stream);
    if (c <= 12288) return launch_norm_shifted<IO, 3, 512>(a, stream);
    if (c <= 16384) return launch_norm_shifted<IO, 2, 1024>(a, stream);
    if (c <= 24576) return launch_norm_shifted<IO, 3, 1024>(a, stream);
    return launch_norm_shifted<IO, 4, 1024>(a, stream);
  }
  if (c <= 1024) return q8_code(launch_after(rmsnorm_q8_single_kernel<IO, 128>, (unsigned)a.rows, 128, 0, stream, 0, a));
  return q8_code(launch_after(rmsnorm_q8_single_kernel<IO, 1024>, (unsigned)a.rows, 1024, 0, stream, 0, a));
}

// ------------------------------------------------------------------ gradient

struct NormGradArgs {
  const void* gy;
  const void* h;
  const void* weight;
  const void* gh;         // may be null
  void* gx;
  void* gw;
  float* part;            // [blocks][cols] partial sums of grad_w
  int64_t rows, ld_gy, ld_h, ld_gh, ld_gx;
  int cols, weight_fp32;
  float eps;
};

// Blocks per SM of the kernel below, of 256 threads: 64 registers per thread with one oct, 128 with two; twice
// that where the elements are 32 bits wide.
template <typename IO>
__host__ __device__ constexpr int group_blocks(int nv) {
  return (nv == 1 ? 4 : 2) * 2 / (int)sizeof(IO);
}

// Asks the L2 for the line of p, a thread's oct: one lane for 128 bytes.
template <typename IO>
__device__ __forceinline__ void prefetch_line(const IO* p) {
  if (threadIdx.x % (16 / sizeof(IO)) == 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}

// grad_w from the blocks' lines of partial sums: WIDTH columns per block and turn, 32 / WIDTH lines per
// warp at a time, all in a fixed order.
template <int THREADS, int WIDTH>
__device__ __forceinline__ void grad_weight_columns(const NormGradArgs& a, int lines) {
  constexpr int kWarps = THREADS / 32, kLines = 32 / WIDTH;
  __shared__ float s[kWarps][WIDTH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int c0 = blockIdx.x * WIDTH; c0 < a.cols; c0 += gridDim.x * WIDTH) {
    const int c = c0 + lane % WIDTH;
    float sum = 0.f;
    if (c < a.cols) {
#pragma unroll 8
      for (int l = warp * kLines + lane / WIDTH; l < lines; l += kWarps * kLines)
        sum += __ldcg(a.part + (int64_t)l * a.cols + c);
    }
#pragma unroll
    for (int k = WIDTH; k < 32; k *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, k);
    if (lane < WIDTH) s[warp][lane] = sum;
    __syncthreads();
    if (threadIdx.x < WIDTH && c < a.cols) {
#pragma unroll
      for (int k = 1; k < kWarps; ++k) sum += s[k][lane];
      if (a.weight_fp32) reinterpret_cast<float*>(a.gw)[c] = sum;
      else reinterpret_cast<__nv_bfloat16*>(a.gw)[c] = __float2bfloat16_rn(sum);
    }
    __syncthreads();
  }
}

// After a barrier of the whole (cooperative) grid: the fewest columns per turn (a sector at least) that
// leave each block one turn, for a block that goes through many lines alone is slow (2048 x 2048: 32
// columns 13.2 us, 8 columns 11.7), and so are several turns (200 x 8192: 11.6 us, with 8 18.5).
template <int THREADS>
__device__ __forceinline__ void grad_weight(const NormGradArgs& a, int rows_per_block = 1) {
  cooperative_groups::this_grid().sync();
  const int lines = (int)min((int64_t)gridDim.x, (a.rows + rows_per_block - 1) / rows_per_block);   // blocks with rows
  if (a.cols <= (int)gridDim.x * 8) grad_weight_columns<THREADS, 8>(a, lines);
  else if (a.cols <= (int)gridDim.x * 16) grad_weight_columns<THREADS, 16>(a, lines);
  else grad_weight_columns<THREADS, 32>(a, lines);
}

// s^3 mean(g h), s last thrice: s^3 alone leaves fp32's range where the row's root mean square is below
// 1e-13 or above 1e13, mean(g h) s does not.
__device__ __forceinline__ float grad_pull(float s, float gh, int cols) { return s * (s * (s * (gh / (float)cols))); }

// The two sums of a row over one oct.
__device__ __forceinline__ void grad_sums(const float2 (&gy)[4], const float2 (&h)[4], const float2 (&w)[4],
                                          float2& ss, float2& gh) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ss = fma2(h[e], h[e], ss);
    gh = fma2(mul2(gy[e], w[e]), h[e], gh);
  }
}
// One oct of grad_x, and of grad_w added to gw.
template <typename IO>
__device__ __forceinline__ void grad_oct(const float2 (&gy)[4], const float2 (&h)[4], const float2 (&w)[4],
                                         const Oct<IO>* add, float s, float k, IO* out, float2 (&gw)[4]) {
  const float2 s2 = make_float2(s, s), nk = make_float2(-k, -k);
  float2 o[4];
  if (add) {
    add->get(o);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fma2(h[e], nk, o[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = mul2(h[e], nk);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 gs = mul2(gy[e], s2);
    gw[e] = fma2(gs, h[e], gw[e]);
    o[e] = fma2(gs, w[e], o[e]);
  }
  Oct<IO> r;
  r.set(o);
  r.store(out);
}

// Two sums over a group of TPR threads; `red`: a word pair per warp, two sets in turn.
template <int TPR>
__device__ __forceinline__ void group_sum2(float& p, float& q, float2* red, int group) {
  p = group_sum<(TPR < 32 ? TPR : 32)>(p);
  q = group_sum<(TPR < 32 ? TPR : 32)>(q);
  if constexpr (TPR > 32) {
    if (threadIdx.x % 32 == 0) red[threadIdx.x % TPR / 32] = make_float2(p, q);
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
    p = q = 0.f;
#pragma unroll
    for (int k = 0; k < TPR / 32; ++k) {
      p += red[k].x;
      q += red[k].y;
    }
  }
}

// Rows up to 4096: a group of TPR threads to a row, 256 / TPR rows per block and turn, the next turn's
// loads in flight while this one is summed; a thread keeps the same columns in all its rows, so its share
// of grad_w stays in registers, and a block's groups add theirs in shared memory.  One cooperative launch:
// the blocks' shares are added behind a grid-wide barrier, which costs less than a second launch.  Heads
// of a query-key norm, 262144 x 128: 52.3 us, 5.1 TB/s, without grad_h 44.1 (a warp per row and block of
// 32: 191).
template <typename IO, typename WT, int NV, int TPR>
__global__ void __launch_bounds__(256, group_blocks<IO>(NV)) rmsnorm_q8_grad_kernel(const NormGradArgs a) {
  constexpr int kRows = 256 / TPR;
  __shared__ __align__(16) float sums[kRows][NV * TPR * 8];
  __shared__ float2 red[2][TPR > 32 ? kRows : 1][TPR > 32 ? TPR / 32 : 1];
  int turn = 0;
  grid_wait();
  grid_trigger();
  const int c0 = (threadIdx.x % TPR) * 8, group = threadIdx.x / TPR;
  const int64_t step = (int64_t)gridDim.x * kRows;
  float2 gw[NV][4];
  Oct<WT> wv[NV];
  Oct<IO> next[NV][3];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      next[v][0].zero();
      next[v][1].zero();
      if (row < a.rows && c < a.cols) {
        next[v][0].load_stream(reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy + c);
        next[v][1].load_stream(reinterpret_cast<const IO*>(a.h) + row * a.ld_h + c);
        if (a.gh) next[v][2].load_stream(reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh + c);
      }
    }
  };
  fetch((int64_t)blockIdx.x * kRows + group);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) gw[v][e] = make_float2(0.f, 0.f);
    wv[v].zero();
    if (c0 + v * TPR * 8 < a.cols) wv[v].load(reinterpret_cast<const WT*>(a.weight) + c0 + v * TPR * 8);
  }
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += step) {
    const int64_t row = base + group;
    Oct<IO> now[NV][3];
    float2 ss2 = make_float2(0.f, 0.f), gh2 = ss2;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int k = 0; k < 3; ++k) now[v][k] = next[v][k];
    fetch(row + step);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float2 gy[4], h[4], w[4];
      now[v][0].get(gy);
      now[v][1].get(h);
      wv[v].get(w);
      grad_sums(gy, h, w, ss2, gh2);
    }
    float ss = ss2.x + ss2.y, gh = gh2.x + gh2.y;
    group_sum2<TPR>(ss, gh, red[turn][TPR > 32 ? group : 0], group);
    turn ^= 1;
    const float s = inv_rms(ss, a.cols, a.eps), k = grad_pull(s, gh, a.cols);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      if (row < a.rows && c < a.cols) {
        float2 gy[4], h[4], w[4];
        now[v][0].get(gy);
        now[v][1].get(h);
        wv[v].get(w);
        grad_oct<IO>(gy, h, w, a.gh ? &now[v][2] : nullptr, s, k, reinterpret_cast<IO*>(a.gx) + row * a.ld_gx + c, gw[v]);
      }
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    Oct<float> o;
    o.set(gw[v]);
    o.store(&sums[group][c0 + v * TPR * 8]);
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.cols && (int64_t)blockIdx.x * kRows < a.rows; c += 256) {
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < kRows; ++g) sum += sums[g][c];
    a.part[(int64_t)blockIdx.x * a.cols + c] = sum;
  }
  grad_weight<256>(a, kRows);
}

// Few rows of 4097 to 8192: as above with a block per row, the next row asked into the L2.
template <typename IO, typename WT, int NV, int TPR>
__global__ void __launch_bounds__(TPR, grad_blocks(TPR, NV)) rmsnorm_q8_grad_wide_kernel(const NormGradArgs a) {
  __shared__ float red[2][64];
  grid_wait();
  grid_trigger();
  const int c0 = threadIdx.x * 8;
  float2 gw[NV][4];
  Oct<WT> wv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) gw[v][e] = make_float2(0.f, 0.f);
    if (c0 + v * TPR * 8 < a.cols) wv[v].load(reinterpret_cast<const WT*>(a.weight) + c0 + v * TPR * 8);
  }
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const IO* gyp = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
    const IO* hp = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
    const IO* ghp = a.gh ? reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh : nullptr;
    Oct<IO> gyv[NV], hv[NV], ghv[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      if (c < a.cols) {
        gyv[v].load_stream(gyp + c);
        hv[v].load_stream(hp + c);
        if (ghp) ghv[v].load_stream(ghp + c);
        if (row + gridDim.x < a.rows) {                          // the row after this one
          prefetch_line(gyp + (int64_t)gridDim.x * a.ld_gy + c);
          prefetch_line(hp + (int64_t)gridDim.x * a.ld_h + c);
          if (ghp) prefetch_line(ghp + (int64_t)gridDim.x * a.ld_gh + c);
        }
      }
    }
    float2 ss2 = make_float2(0.f, 0.f), gh2 = ss2;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (c0 + v * TPR * 8 < a.cols) {
        float2 gy[4], h[4], w[4];
        gyv[v].get(gy);
        hv[v].get(h);
        wv[v].get(w);
        grad_sums(gy, h, w, ss2, gh2);
      }
    }
    float ss = ss2.x + ss2.y, gh = gh2.x + gh2.y;
    block_sum2<TPR>(ss, gh, red[turn]);
    const float s = inv_rms(ss, a.cols, a.eps), k = grad_pull(s, gh, a.cols);
    IO* gxp = reinterpret_cast<IO*>(a.gx) + row * a.ld_gx;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      if (c < a.cols) {
        float2 gy[4], h[4], w[4];
        gyv[v].get(gy);
        hv[v].get(h);
        wv[v].get(w);
        grad_oct<IO>(gy, h, w, ghp ? &ghv[v] : nullptr, s, k, gxp + c, gw[v]);
      }
    }
  }
  float* part = a.part + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int v = 0; v < NV && blockIdx.x < a.rows; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < a.cols) {
      Oct<float> o;
      o.set(gw[v]);
      o.store(part + c);
    }
  }
  grad_weight<TPR>(a);
}

// Large matrices: rows streamed through a ring, all 16 warps to a row (narrower rows go by groups of
// threads, run_grad), so that a thread's share of grad_w is the block's.
template <typename IO, typename WT, bool GH>
__global__ void __launch_bounds__(kRingThreads, 1)
rmsnorm_q8_grad_stream_kernel(const NormGradArgs a, int stages, int* status) {
  constexpr int kArr = GH ? 3 : 2, kNV = 2, kR = kRingRows<IO>, W = kRingWarps, kStep = W * 32 * 8;
  const int c0 = (threadIdx.x % (W * 32)) * 8;
  const void* const src[3] = {a.gy, a.h, a.gh};
  const int64_t ld[3] = {a.ld_gy, a.ld_h, a.ld_gh};
  RowRing<IO, W, kR, kArr> ring(ring_block<W, kR>(), src, ld, a.rows, a.cols, stages, status);
  float2 gw[kNV][4], w[kNV][4];
#pragma unroll
  for (int v = 0; v < kNV; ++v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) gw[v][e] = make_float2(0.f, 0.f);
    if (c0 + v * kStep < a.cols) load_oct(reinterpret_cast<const WT*>(a.weight) + c0 + v * kStep, w[v]);
  }
  ring.start();
  if (ring.producer) ring.serve();
  const int n = ring.producer ? 0 : ring.n;
  for (int i = 0; i < n; ++i) {
    const int64_t row = ring.row(i);
    const int high = ring.height(i);
    float2 gy[kR][kNV][4];                // h is read again: both would spill
    float ss[kR], gh[kR];
#pragma unroll
    for (int r = 0; r < kR; ++r) ss[r] = gh[r] = 0.f;
    if (ring.wait()) {
#pragma unroll
      for (int r = 0; r < kR; ++r) {
        if (r < high) {
          float2 ss2 = make_float2(0.f, 0.f), gh2 = ss2;
#pragma unroll
          for (int v = 0; v < kNV; ++v) {
            const int c = c0 + v * kStep;
            if (c < a.cols) {
              float2 h[4];
              load_oct(ring.at(r, 0) + c, gy[r][v]);
              load_oct(ring.at(r, 1) + c, h);
              grad_sums(gy[r][v], h, w[v], ss2, gh2);
            }
          }
          ss[r] = ss2.x + ss2.y;
          gh[r] = gh2.x + gh2.y;
        }
      }
    }
    ring.template reduce<true>(i, ss, gh);
    if (ring.ok) {
#pragma unroll
      for (int r = 0; r < kR; ++r) {
        if (r < high) {
          const float s = inv_rms(ss[r], a.cols, a.eps), k = grad_pull(s, gh[r], a.cols);
          IO* gxp = reinterpret_cast<IO*>(a.gx) + (row + r) * a.ld_gx;
#pragma unroll
          for (int v = 0; v < kNV; ++v) {
            const int c = c0 + v * kStep;
            if (c < a.cols) {
              Oct<IO> add;
              float2 h[4];
              load_oct(ring.at(r, 1) + c, h);
              if constexpr (GH) add.load(ring.at(r, 2) + c);
              grad_oct<IO>(gy[r][v], h, w[v], GH ? &add : nullptr, s, k, gxp + c, gw[v]);
            }
          }
        }
      }
    }
    ring.release();
    ring.advance();
  }
  ring.finish();
#pragma unroll
  for (int v = 0; v < kNV; ++v) {
    const int c = c0 + v * kStep;
    if (!ring.producer && c < a.cols) {
      Oct<float> o;
      o.set(gw[v]);
      o.store(a.part + (int64_t)blockIdx.x * a.cols + c);
    }
  }
  grad_weight<kRingThreads>(a);
}

// Rows that start anywhere, or too wide for the kernels above.  The grid is a multiple of eight blocks
// (or has one row per block: grad_shifted_grid), so that all rows of a block start alike and a thread keeps
// its columns.
template <typename IO, int NV, int TPR>
__global__ void __launch_bounds__(TPR, grad_blocks(TPR, NV)) rmsnorm_q8_grad_shifted_kernel(const NormGradArgs a) {
  __shared__ float red[2][64];
  const int shift = oct_shift(reinterpret_cast<const IO*>(a.h) + (int64_t)blockIdx.x * a.ld_h);
  float2 gw[NV][4], w[NV][4];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    load_factors(a.weight, a.weight_fp32, ((int)threadIdx.x + v * TPR) * 8 - shift, a.cols, w[v]);
#pragma unroll
    for (int e = 0; e < 4; ++e) gw[v][e] = make_float2(0.f, 0.f);
  }
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const OctRow<IO> gyr(a.gy, row, a.rows, a.ld_gy, a.cols), hr(a.h, row, a.rows, a.ld_h, a.cols),
        ghr(a.gh ? a.gh : a.h, row, a.rows, a.gh ? a.ld_gh : a.ld_h, a.cols);
    Oct<IO> gyv[NV], hv[NV], ghv[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = ((int)threadIdx.x + v * TPR) * 8 - shift;
      gyr.load(c, a.cols, gyv[v]);
      hr.load(c, a.cols, hv[v]);
      if (a.gh) ghr.load(c, a.cols, ghv[v]);
      if (row + gridDim.x < a.rows && c >= 0 && c < a.cols) {     // the row after this one
        prefetch_line(gyr.p + (int64_t)gridDim.x * a.ld_gy + c);
        prefetch_line(hr.p + (int64_t)gridDim.x * a.ld_h + c);
        if (a.gh) prefetch_line(ghr.p + (int64_t)gridDim.x * a.ld_gh + c);
      }
    }
    float2 ss2 = make_float2(0.f, 0.f), gh2 = ss2;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = ((int)threadIdx.x + v * TPR) * 8 - shift;
      float2 gy[4], h[4];
      get_part(gyv[v], c, a.cols, gy);
      get_part(hv[v], c, a.cols, h);
      grad_sums(gy, h, w[v], ss2, gh2);
    }
    float ss = ss2.x + ss2.y, gh = gh2.x + gh2.y;
    block_sum2<TPR>(ss, gh, red[turn]);
    const float s = inv_rms(ss, a.cols, a.eps), k = grad_pull(s, gh, a.cols);
    const float2 s2 = make_float2(s, s), nk = make_float2(-k, -k);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = ((int)threadIdx.x + v * TPR) * 8 - shift;
      float2 gy[4], h[4], o[4];
      get_part(gyv[v], c, a.cols, gy);
      get_part(hv[v], c, a.cols, h);
      if (a.gh) {
        ghv[v].get(o);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 gs = mul2(gy[e], s2);
        gw[v][e] = fma2(gs, h[e], gw[v][e]);
        o[e] = fma2(gs, w[v][e], fma2(h[e], nk, o[e]));
      }
      store_part(reinterpret_cast<IO*>(a.gx) + row * a.ld_gx, c, a.cols, o);
    }
  }
  float* part = a.part + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int v = 0; v < NV && blockIdx.x < a.rows; ++v) {
    const int c = ((int)threadIdx.x + v * TPR) * 8 - shift;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c + k >= 0 && c + k < a.cols) part[c + k] = k & 1 ? gw[v][k / 2].y : gw[v][k / 2].x;
  }
  grad_weight<TPR>(a);
}

// Any alignment, any length: two passes over the row, and the block's share of grad_w collected in
// its line of the scratch (each thread its own columns).
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS, grad_blocks(THREADS)) rmsnorm_q8_grad_single_kernel(const NormGradArgs a) {
  __shared__ float red[2][64];
  grid_wait();
  grid_trigger();
  float* part = a.part + (int64_t)blockIdx.x * a.cols;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const IO* gyp = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
    const IO* hp = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
    const IO* ghp = a.gh ? reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh : nullptr;
    IO* gxp = reinterpret_cast<IO*>(a.gx) + row * a.ld_gx;
    float ss = 0.f, gh = 0.f;
#pragma unroll 4
    for (int c = threadIdx.x; c < a.cols; c += THREADS) {
      const float h = to_f32(hp[c]);
      ss += h * h;
      gh += to_f32(gyp[c]) * load1(a.weight, a.weight_fp32, c) * h;
    }
    block_sum2<THREADS>(ss, gh, red[turn]);
    const float s = inv_rms(ss, a.cols, a.eps), k = grad_pull(s, gh, a.cols);
#pragma unroll 4
    for (int c = threadIdx.x; c < a.cols; c += THREADS) {
      const float h = to_f32(hp[c]), gy = to_f32(gyp[c]);
      float out = s * (gy * load1(a.weight, a.weight_fp32, c)) - h * k;
      if (ghp) out += to_f32(ghp[c]);
      from_f32(gxp + c, out);
      const float add = gy * h * s;
      part[c] = row == (int64_t)blockIdx.x ? add : part[c] + add;
    }
  }
  grad_weight<THREADS>(a);
}

template <typename IO, typename WT, bool GH>
int launch_grad_stream(const NormGradArgs& a, cudaStream_t stream) {
  constexpr int kR = kRingRows<IO>;
  static PerDeviceOnce once;
  return launch_ring(rmsnorm_q8_grad_stream_kernel<IO, WT, GH>, once, (unsigned)ring_grid(a.rows, kR, 1, 1, q8_sms()),
                     (size_t)a.cols * sizeof(IO) * (GH ? 3 : 2) * kR, 0, stream, a);
}
int launch_grad_grid(void (*kernel)(NormGradArgs), NormGradArgs a, int threads, int64_t grid, cudaStream_t stream) {
  void* args[1] = {&a};
  return q8_code(cudaLaunchCooperativeKernel((const void*)kernel, dim3((unsigned)grid), dim3((unsigned)threads), args, 0,
                                             stream));
}
int launch_grad(void (*kernel)(NormGradArgs), const NormGradArgs& a, int threads, int nv, cudaStream_t stream) {
  return launch_grad_grid(kernel, a, threads, grad_grid(a.rows, a.cols, grad_blocks(threads, nv), q8_sms()), stream);
}
template <typename IO, typename WT, int NV, int TPR>
int launch_grad_groups(const NormGradArgs& a, cudaStream_t stream) {
  constexpr int kRows = 256 / TPR;
  const int sms = q8_sms();
  const int64_t blocks = std::min<int64_t>((a.rows + kRows - 1) / kRows, group_blocks<IO>(NV) * sms);
  return launch_grad_grid(rmsnorm_q8_grad_kernel<IO, WT, NV, TPR>, a, 256, grad_grid_for_columns(blocks, a.cols, sms),
                          stream);
}

template <typename IO, typename WT>
int run_grad(const NormGradArgs& a, cudaStream_t stream) {
  const int c = a.cols;
  if (c <= 64) return launch_grad_groups<IO, WT, 1, 8>(a, stream);
  if (c <= 128) return launch_grad_groups<IO, WT, 1, 16>(a, stream);
  if (c <= 256) return launch_grad_groups<IO, WT, 1, 32>(a, stream);
  if (c <= 512) return launch_grad_groups<IO, WT, 2, 32>(a, stream);
  if (c <= 1024) return launch_grad_groups<IO, WT, 2, 64>(a, stream);
  if (c <= 2048) return launch_grad_groups<IO, WT, 2, 128>(a, stream);
  if (c <= 4096) return launch_grad_groups<IO, WT, 2, 256>(a, stream);
  // Streamed from these sizes on (8192 x 5120: 72 us, a block per row 106, in fp32 113 and 154), else a row or
  // two per block (100 x 8192: 10.4 us).  Up to 4096 columns the ring is little faster than groups (8192 x
  // 4096: 50.9 us against 52.3) or slower (2048 x 2048: 14.8 against 11.4).
  if (a.rows * c < (int64_t)1 << 21) return launch_grad(rmsnorm_q8_grad_wide_kernel<IO, WT, 2, 512>, a, 512, 2, stream);
  return a.gh ? launch_grad_stream<IO, WT, true>(a, stream) : launch_grad_stream<IO, WT, false>(a, stream);
}

// `alike`: the matrices' rows start alike.
template <typename IO>
int run_grad_single(const NormGradArgs& a, bool alike, cudaStream_t stream) {
  const GradForm form = alike ? grad_shifted_form(a.cols) : GradForm{0, 0};
  auto go = [&](auto kernel) {
    return launch_grad_grid(kernel, a, form.threads, grad_shifted_grid(a.rows, a.cols, form, q8_sms()), stream);
  };
  switch (form.threads) {
    case 32: return go(rmsnorm_q8_grad_shifted_kernel<IO, 1, 32>);
    case 128: return go(rmsnorm_q8_grad_shifted_kernel<IO, 1, 128>);
    case 256:
      return form.nv == 1   ? go(rmsnorm_q8_grad_shifted_kernel<IO, 1, 256>)
             : form.nv == 2 ? go(rmsnorm_q8_grad_shifted_kernel<IO, 2, 256>)
                            : go(rmsnorm_q8_grad_shifted_kernel<IO, 3, 256>);
    case 512: return go(rmsnorm_q8_grad_shifted_kernel<IO, 2, 512>);
    case 1024: return go(rmsnorm_q8_grad_shifted_kernel<IO, 2, 1024>);
  }
  if (a.cols <= 1024) return launch_grad(rmsnorm_q8_grad_single_kernel<IO, 128>, a, 128, 1, stream);
  return launch_grad(rmsnorm_q8_grad_single_kernel<IO, 1024>, a, 1024, 1, stream);
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
  const NormArgs a = {x,    residual,    weight, h_out, (uint8_t*)q_out, scale_out, rows,
                      ld_x, ld_residual, ld_h,   ld_q,  (int)cols,       weight_fp32, format, eps};
  const bool octs = cols % 8 == 0 && cols <= 16384 && ld_x % 8 == 0 && ld_q % 8 == 0 && aligned16(x) &&
                    aligned16(weight) && ((uintptr_t)q_out & 7) == 0 &&
                    (!residual || (ld_residual % 8 == 0 && ld_h % 8 == 0 && aligned16(residual) && aligned16(h_out)));
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (!octs) {
    auto alike = [&](auto type) {
      using T = decltype(type);
      return ((uintptr_t)q_out & 7) == 0 && ld_q % 8 == 0 &&
             (!residual || (octs_alike<T>(x, ld_x, residual, ld_residual) && octs_alike<T>(x, ld_x, h_out, ld_h)));
    };
    return io_fp32 ? run_norm_single<float>(a, alike(float()), stream)
                   : run_norm_single<__nv_bfloat16>(a, alike(__nv_bfloat16()), stream);
  }
  if (io_fp32) return weight_fp32 ? run_norm<float, float>(a, stream) : run_norm<float, __nv_bfloat16>(a, stream);
  return weight_fp32 ? run_norm<__nv_bfloat16, float>(a, stream) : run_norm<__nv_bfloat16, __nv_bfloat16>(a, stream);
}

extern "C" size_t prm_rmsnorm_q8_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1) return 0;
  return (size_t)grad_parts(rows, cols) * (size_t)cols * 4;
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
    return q8_code(cudaMemsetAsync(grad_weight, 0, (size_t)cols * (weight_fp32 ? 4 : 2), stream));
  if (!grad_y || !h || !weight || !grad_x || !scratch) return PRM_ERR_ARG;
  if (scratch_bytes < prm_rmsnorm_q8_scratch_bytes(rows, cols)) return PRM_ERR_WORKSPACE;
  const int es = io_fp32 ? 4 : 2;
  if (((uintptr_t)grad_y | (uintptr_t)h | (uintptr_t)grad_h | (uintptr_t)grad_x) % es != 0 ||
      (uintptr_t)weight % (weight_fp32 ? 4 : 2) != 0 || ((uintptr_t)scratch & 15) != 0)
    return PRM_ERR_ALIGN;
  const NormGradArgs a = {grad_y, h,         weight, grad_h,    grad_x,    grad_weight, (float*)scratch, rows,
                          ld_grad_y, ld_h,   ld_grad_h, ld_grad_x, (int)cols, weight_fp32, eps};
  const bool octs = cols % 8 == 0 && cols <= 8192 && ld_grad_y % 8 == 0 && ld_h % 8 == 0 && ld_grad_x % 8 == 0 &&
                    aligned16(grad_y) && aligned16(h) && aligned16(grad_x) && aligned16(weight) &&
                    (!grad_h || (ld_grad_h % 8 == 0 && aligned16(grad_h)));
  if (!octs) {
    auto alike = [&](auto type) {
      using T = decltype(type);
      return octs_alike<T>(h, ld_h, grad_y, ld_grad_y) && octs_alike<T>(h, ld_h, grad_x, ld_grad_x) &&
             (!grad_h || octs_alike<T>(h, ld_h, grad_h, ld_grad_h));
    };
    return io_fp32 ? run_grad_single<float>(a, alike(float()), stream)
                   : run_grad_single<__nv_bfloat16>(a, alike(__nv_bfloat16()), stream);
  }
  if (io_fp32) return weight_fp32 ? run_grad<float, float>(a, stream) : run_grad<float, __nv_bfloat16>(a, stream);
  return weight_fp32 ? run_grad<__nv_bfloat16, float>(a, stream) : run_grad<__nv_bfloat16, __nv_bfloat16>(a, stream);
}
