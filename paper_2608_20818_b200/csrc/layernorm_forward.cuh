// Kernels of the layer norm's forward pass; layernorm.cu has those of aligned rows, layernorm_shifted.cu those
// of rows that start anywhere (apart only to be compiled side by side).
#pragma once

#include "layernorm.cuh"

namespace prm {

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
  uint32_t rows_per_block_y;   // of the launch: 0, or rows_per_group where blockIdx.y is the group
  int divide;                  // the group of a row has to be computed
  float eps, over;         // over: 1 / cols
  Affine affine;
  Drop drop;
};

// By the stream's type.
int layernorm_aligned(const LayerNormArgs& a, const __nv_bfloat16*, cudaStream_t stream);
int layernorm_aligned(const LayerNormArgs& a, const float*, cudaStream_t stream);
int layernorm_shifted(const LayerNormArgs& a, const __nv_bfloat16*, cudaStream_t stream);
int layernorm_shifted(const LayerNormArgs& a, const float*, cudaStream_t stream);

namespace {

// What the row's numbers are: mean and rstd, and what is still to be taken off h - (first mean).
struct RowStats {
  float mean, rstd, rest;
  // of the first mean, the sums of h - mean and of its squares.  An infinity among the row's elements leaves the mean
  // infinite and rstd NaN, a NaN both; infinite squares of finite elements leave rstd 0 (rest^2 may be as large).
  __device__ __forceinline__ RowStats(float first, float2 sums, float over, float eps) {
    rest = sums.x * over;
    mean = fabsf(first) < INFINITY ? first + rest : first;
    const float square = sums.y * over, var = square < INFINITY ? square - rest * rest : square;
    rstd = rsqrtf((var < 0.f ? 0.f : var) + eps);
  }
};

// Sums, statistics and output of a row that a group of TPR threads holds in t (zeros outside the row; `in`: whether an
// oct lies in it).  Threads beyond the row compute on zeros: a branch around each oct costs more.
template <int NV, int TPR, int BLOCK, bool SHIFT>
__device__ __forceinline__ RowStats row_stats(float2 (&t)[NV][4], const bool (&in)[NV], int c0, int cols, float over, float eps,
                                              float* red, float* red2) {
  float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum2 = add2(sum2, t[v][e]);
  float sum[1] = {sum2.x + sum2.y}, both[2] = {0.f, 0.f};
  row_sums<TPR, BLOCK>(sum, red);
  sum[0] *= over;
  const float2 off2 = make_float2(-sum[0], -sum[0]);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    float2 dev2 = make_float2(0.f, 0.f), square2 = dev2;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[v][e] = add2(t[v][e], off2);
    if constexpr (SHIFT) clear_outside(c0 + v * TPR * 8, cols, t[v]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dev2 = add2(dev2, t[v][e]);
      square2 = fma2(t[v][e], t[v][e], square2);
    }
    both[0] += in[v] ? dev2.x + dev2.y : 0.f;
    both[1] += in[v] ? square2.x + square2.y : 0.f;
  }
  row_sums<TPR, BLOCK>(both, red2);
  return RowStats(sum[0], make_float2(both[0], both[1]), over, eps);
}

// Blocks per SM of the kernel for many rows: 64 registers per thread, 80 and more for wide rows (8192 x 4096 with dropout: 5 us
// more with 64 registers; 131072 x 128 without: 2 us less).
constexpr int layernorm_blocks(int tpr, int block) { return tpr >= 256 ? 768 / block : 1024 / block; }

// Few rows: one for each group of TPR threads, BLOCK / TPR rows per block, 8 * NV elements per thread.  SHIFT: octs
// aligned in memory, of rows that start anywhere.
template <typename IO, int NV, int TPR, int BLOCK, bool DROP, bool SHIFT>
__global__ void __launch_bounds__(BLOCK) layernorm_kernel(const LayerNormArgs a) {
  constexpr int kLines = BLOCK / TPR;
  constexpr bool EARLY = !SHIFT && NV <= 2;                     // weights are fetched along with the row
  __shared__ __align__(16) float red[kLines][TPR > 32 ? TPR / 32 : 4];
  __shared__ __align__(16) float red2[kLines][TPR > 32 ? TPR / 32 * 2 : 4];
  grid_wait();
  grid_trigger();
  const int line = threadIdx.x / TPR;
  // Blocks of a group's rows (blockIdx.y: the group), or of all rows.
  const uint32_t first_row = blockIdx.y * a.rows_per_block_y, in_group = blockIdx.x * kLines + line;
  const uint32_t limit = a.rows_per_block_y ? a.rows_per_block_y : (uint32_t)a.rows;
  const int64_t row0 = first_row + min(in_group, limit - 1);
  uint32_t group = blockIdx.y;
  if (a.divide) group = (uint32_t)row0 / a.rows_per_group;
  const IO* xp = reinterpret_cast<const IO*>(a.x) + row0 * a.ld_x;
  const int shift = SHIFT ? oct_shift(xp) : 0;
  const int c0 = (int)(threadIdx.x % TPR) * 8 - shift;
  const bool live = in_group < limit;
  bool in[NV];                                                  // the row is one, and the thread's octs lie in it
#pragma unroll
  for (int v = 0; v < NV; ++v) in[v] = live && c0 + v * TPR * 8 < a.cols;
  Oct<IO> xv[NV], rv[NV];
  RawFactors wv[EARLY ? NV : 1], bv[EARLY ? NV : 1];
  if constexpr (SHIFT) {
    const OctRow<IO> x(a.x, row0, a.rows, a.ld_x, a.cols);
    const OctRow<IO> res(a.residual ? a.residual : a.x, row0, a.rows, a.residual ? a.ld_r : a.ld_x, a.cols);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      x.load(c, live ? a.cols : 0, xv[v]);
      if (a.residual) res.load(c, live ? a.cols : 0, rv[v]);
    }
  } else {
    xp += c0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      xv[v].zero();
      if (in[v]) xv[v].load_stream(xp + v * TPR * 8);
    }
    if (a.residual) {
      const IO* rp = reinterpret_cast<const IO*>(a.residual) + row0 * a.ld_r + c0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        rv[v].zero();
        if (in[v]) rv[v].load_stream(rp + v * TPR * 8);
      }
    }
  }
  auto fetch_affine = [&](int v, RawFactors& w, RawFactors& b) {
    const int c = in[v] ? c0 + v * TPR * 8 : 0;
    if (a.affine.weight) w.load(a.affine.weight, a.affine.fp32, group * a.affine.ld_w + c);
    if (a.affine.bias) b.load(a.affine.bias, a.affine.fp32, group * a.affine.ld_b + c);
  };
  if constexpr (EARLY) {
#pragma unroll
    for (int v = 0; v < NV; ++v) fetch_affine(v, wv[v], bv[v]);
  }
  const uint64_t number = DROP ? drop_number(a.drop) : 0;
  IO* h = reinterpret_cast<IO*>(a.h) + row0 * a.ld_h;
  float2 t[NV][4];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if constexpr (SHIFT) get_part(xv[v], c, a.cols, t[v]);
    else xv[v].get(t[v]);
    if constexpr (DROP) drop_oct<!SHIFT>(a.drop, number, (uint32_t)row0, c, t[v]);
    if (a.residual) {
      float2 add[4];
      if constexpr (SHIFT) get_part(rv[v], c, a.cols, add);
      else rv[v].get(add);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[v][e] = add2(t[v][e], add[e]);
    }
    if (a.h) {
      Oct<IO> o;
      o.set(t[v]);
      o.get(t[v]);                                              // as it is stored
      if (in[v]) {
        if constexpr (SHIFT) store_part(h, c, a.cols, t[v]);
        else o.store(h + c);
      }
    }
  }
  const RowStats s = row_stats<NV, TPR, BLOCK, SHIFT>(t, in, c0, a.cols, a.over, a.eps, red[line], red2[line]);
  const float2 rs2 = make_float2(s.rstd, s.rstd), rest2 = make_float2(-s.rest * s.rstd, -s.rest * s.rstd);
  const float one = a.affine.add_one ? 1.f : 0.f;
  IO* y = reinterpret_cast<IO*>(a.y) + row0 * a.ld_y;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    float2 w[4], b[4];
    if constexpr (SHIFT) {
      affine_weight(a.affine, group, c, a.cols, w);
      affine_bias(a.affine, group, c, a.cols, b);
    } else {
      if constexpr (!EARLY) fetch_affine(v, wv[0], bv[0]);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = make_float2(1.f, 1.f), b[e] = make_float2(0.f, 0.f);
      if (a.affine.weight) {
        wv[EARLY ? v : 0].get(a.affine.fp32, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = add2(w[e], make_float2(one, one));
      }
      if (a.affine.bias) bv[EARLY ? v : 0].get(a.affine.fp32, b);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) t[v][e] = fma2(fma2(t[v][e], rs2, rest2), w[e], b[e]);
    if (in[v]) {
      if constexpr (SHIFT) {
        store_part(y, c, a.cols, t[v]);
      } else {
        Oct<IO> o;
        o.set(t[v]);
        o.store(y + c);
      }
    }
  }
  if (threadIdx.x % TPR == 0 && live) {
    a.mean[row0] = s.mean;
    a.rstd[row0] = s.rstd;
  }
}

// The words that hold weight and bias of a group in shared memory.
__host__ __device__ inline int staged_words(int cols, bool shift) {
  const int octs = (cols + 7) / 8;
  return shift ? 2 * (octs * 8 + octs / 4 + 1) : octs * 16;
}

// Many rows: a block's rows are a range, BLOCK / TPR of them at a time, the next rows' loads under way while these are summed.
// The rows of a group share weight and bias from shared memory, as fp32: fetched by each row for itself they cost as many
// bytes from L2 as the row, and their conversion (16384 x 2048 with a weight for each of 64 groups, no residual: 29
// us, 4.7 TB/s; a row per block some 10 more).  Asking the L2 for the rows after the next gains nothing here.  ROUND: one group, whose rows go
// round the blocks, so that rows under way at a time are neighbours (8192 x 4096 with dropout: 55 us, 8192 x 8192 94; in ranges 4 more each).
template <typename IO, int NV, int TPR, int BLOCK, bool DROP, bool SHIFT, bool ROUND>
__global__ void __launch_bounds__(BLOCK, layernorm_blocks(TPR, BLOCK)) layernorm_many_kernel(const LayerNormArgs a) {
  constexpr int kLines = BLOCK / TPR;
  extern __shared__ __align__(16) float staged[];
  __shared__ __align__(16) float red[kLines][TPR > 32 ? TPR / 32 : 4];
  __shared__ __align__(16) float red2[kLines][TPR > 32 ? TPR / 32 * 2 : 4];
  grid_wait();
  grid_trigger();
  const int line = threadIdx.x / TPR, octs = (a.cols + 7) / 8, half = staged_words(a.cols, SHIFT) / 2;
  const int64_t r0 = ROUND ? (int64_t)blockIdx.x * kLines : a.rows * blockIdx.x / gridDim.x;
  const int64_t r1 = ROUND ? a.rows : a.rows * (blockIdx.x + 1) / gridDim.x, step = ROUND ? (int64_t)gridDim.x * kLines : kLines;
  const uint64_t number = DROP ? drop_number(a.drop) : 0;
  const float one = a.affine.add_one ? 1.f : 0.f;
  Oct<IO> xv[NV], rv[NV];
  int shift = 0;                                                // of the row in xv
  bool in[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) in[v] = ((int)(threadIdx.x % TPR) + v * TPR) * 8 < a.cols;
  auto fetch = [&](int64_t row, int64_t end) {
    if (row >= end) return;
    if constexpr (SHIFT) {
      const OctRow<IO> x(a.x, row, a.rows, a.ld_x, a.cols);
      const OctRow<IO> r(a.residual ? a.residual : a.x, row, a.rows, a.residual ? a.ld_r : a.ld_x, a.cols);
      shift = oct_shift(x.p);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = ((int)(threadIdx.x % TPR) + v * TPR) * 8 - shift;
        x.load(c, a.cols, xv[v]);
        if (a.residual) r.load(c, a.cols, rv[v]);
      }
    } else {
      const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x + threadIdx.x % TPR * 8;
      const IO* r = reinterpret_cast<const IO*>(a.residual) + row * a.ld_r + threadIdx.x % TPR * 8;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (in[v]) xv[v].load_stream(x + v * TPR * 8);
      if (a.residual) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
          if (in[v]) rv[v].load_stream(r + v * TPR * 8);
      }
    }
  };
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    xv[v].zero();
    rv[v].zero();
  }
  for (int64_t begin = r0; begin < r1;) {
    const uint32_t group = ROUND ? 0u : (uint32_t)begin / a.rows_per_group;
    const int64_t end = ROUND ? r1 : min(r1, (int64_t)(group + 1) * a.rows_per_group);
    fetch(begin + line, end);
    if (!ROUND && begin > r0) __syncthreads();                            // the group before has been read
    // aligned octs: the first halves of all, then the second halves, so that neighbours read neighbouring 16 bytes;
    // else single words, 33 apart for 32 (neighbours read words that are 8 apart)
    for (int o = threadIdx.x; o < octs; o += BLOCK) {
      float2 w[4], b[4];
      affine_weight(a.affine, group, o * 8, a.cols, w);
      affine_bias(a.affine, group, o * 8, a.cols, b);
      if constexpr (SHIFT) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = o * 8 + k + o / 4;
          staged[at] = k & 1 ? w[k / 2].y : w[k / 2].x;
          staged[half + at] = k & 1 ? b[k / 2].y : b[k / 2].x;
        }
      } else {
        float4* s = reinterpret_cast<float4*>(staged) + o;
        s[0] = make_float4(w[0].x, w[0].y, w[1].x, w[1].y);
        s[octs] = make_float4(w[2].x, w[2].y, w[3].x, w[3].y);
        s[2 * octs] = make_float4(b[0].x, b[0].y, b[1].x, b[1].y);
        s[3 * octs] = make_float4(b[2].x, b[2].y, b[3].x, b[3].y);
      }
    }
    __syncthreads();
    for (int64_t base = begin; base < end; base += step) {
      const int64_t row = base + line;
      const bool live = row < end;
      const int c0 = (int)(threadIdx.x % TPR) * 8 - shift;
      float2 t[NV][4];
      Oct<IO> res[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * TPR * 8;
        if constexpr (SHIFT) {
          get_part(xv[v], c, a.cols, t[v]);
          in[v] = c < a.cols;
        } else {
          xv[v].get(t[v]);
        }
        res[v] = rv[v];
      }
      fetch(row + step, end);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * TPR * 8;
        if constexpr (DROP) drop_oct<!SHIFT>(a.drop, number, (uint32_t)row, c, t[v]);
        if (a.residual) {
          float2 add[4];
          if constexpr (SHIFT) get_part(res[v], c, a.cols, add);
          else res[v].get(add);
#pragma unroll
          for (int e = 0; e < 4; ++e) t[v][e] = add2(t[v][e], add[e]);
        }
        if (a.h) {
          IO* h = reinterpret_cast<IO*>(a.h) + row * a.ld_h;
          Oct<IO> o;
          o.set(t[v]);
          o.get(t[v]);                                          // as it is stored
          if (in[v] && live) {
            if constexpr (SHIFT) store_part(h, c, a.cols, t[v]);
            else o.store(h + c);
          }
        }
      }
      const RowStats s = row_stats<NV, TPR, BLOCK, SHIFT>(t, in, c0, a.cols, a.over, a.eps, red[line], red2[line]);
      const float2 rs2 = make_float2(s.rstd, s.rstd), rest2 = make_float2(-s.rest * s.rstd, -s.rest * s.rstd);
      IO* y = reinterpret_cast<IO*>(a.y) + row * a.ld_y;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * TPR * 8;
        float2 w[4], b[4];
        if constexpr (SHIFT) {
          float f[16];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int e = min(max(c + k, 0), a.cols - 1), at = e + e / 32;
            f[k] = staged[at];
            f[8 + k] = staged[half + at];
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = make_float2(f[2 * e], f[2 * e + 1]);
            b[e] = make_float2(f[8 + 2 * e], f[8 + 2 * e + 1]);
          }
        } else {
          const float4* f = reinterpret_cast<const float4*>(staged) + (in[v] ? c / 8 : 0);
          const float4 w0 = f[0], w1 = f[octs], b0 = f[2 * octs], b1 = f[3 * octs];
          w[0] = make_float2(w0.x, w0.y), w[1] = make_float2(w0.z, w0.w), w[2] = make_float2(w1.x, w1.y), w[3] = make_float2(w1.z, w1.w);
          b[0] = make_float2(b0.x, b0.y), b[1] = make_float2(b0.z, b0.w), b[2] = make_float2(b1.x, b1.y), b[3] = make_float2(b1.z, b1.w);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) t[v][e] = fma2(fma2(t[v][e], rs2, rest2), w[e], b[e]);
        if (in[v] && live) {
          if constexpr (SHIFT) {
            store_part(y, c, a.cols, t[v]);
          } else {
            Oct<IO> o;
            o.set(t[v]);
            o.store(y + c);
          }
        }
      }
      if (threadIdx.x % TPR == 0 && live) {
        a.mean[row] = s.mean;
        a.rstd[row] = s.rstd;
      }
    }
    begin = end;
  }
}

// Any alignment, any length: three passes over the row, four elements per thread at a time, the later two of
// what the thread wrote itself (or of x).
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS) layernorm_single_kernel(const LayerNormArgs a) {
  __shared__ __align__(16) float red[THREADS / 32];
  __shared__ __align__(16) float red2[THREADS / 32 * 2];
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
  float total[1] = {sum};
  row_sums<THREADS, THREADS>(total, red);
  const float first = total[0] * a.over;
  const IO* src = h ? h : x;
  float sums[2] = {0.f, 0.f};
  for (int c = threadIdx.x * 4; c < a.cols; c += THREADS * 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (c + k < a.cols) {
        const float v = to_f32(src[c + k]) - first;
        sums[0] += v;
        sums[1] += v * v;
      }
    }
  }
  row_sums<THREADS, THREADS>(sums, red2);
  const RowStats s(first, make_float2(sums[0], sums[1]), a.over, a.eps);
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

template <typename IO>
int run_layernorm_single(const LayerNormArgs& a, cudaStream_t stream) {
  if (a.cols <= 1024) return q8_code(launch_after(layernorm_single_kernel<IO, 128>, (unsigned)a.rows, 128, 0, stream, 0, a));
  return q8_code(launch_after(layernorm_single_kernel<IO, 1024>, (unsigned)a.rows, 1024, 0, stream, 0, a));
}
template <typename IO, bool DROP, bool SHIFT, int NV, int TPR>
int launch_layernorm(LayerNormArgs a, cudaStream_t stream) {
  constexpr int BLOCK = TPR < 256 ? 256 : TPR, kRows = BLOCK / TPR;
  // A block per kRows rows of a group; groups of fewer rows than that share blocks, and each row looks its own up.
  const bool by_group = a.rows_per_group < a.rows && a.rows_per_group >= kRows && a.rows % a.rows_per_group == 0 &&
                        a.rows / a.rows_per_group <= 65535;
  const int64_t rows = by_group ? a.rows_per_group : a.rows;
  a.rows_per_block_y = by_group ? a.rows_per_group : 0;
  a.divide = a.rows_per_group < a.rows && !by_group;
  return q8_code(launch_after(layernorm_kernel<IO, NV, TPR, BLOCK, DROP, SHIFT>,
                              dim3((unsigned)((rows + kRows - 1) / kRows), by_group ? (unsigned)(a.rows / rows) : 1u),
                              BLOCK, 0, stream, 0, a));
}
// (bf16 only: 32-bit elements leave room for fewer rows under way; 8192 x 4096 with residual 84 us with a block per row, so 15 more.)
template <typename IO, bool DROP, bool SHIFT, int NV, int TPR, bool ROUND>
int launch_layernorm_many_as(const LayerNormArgs& a, cudaStream_t stream) {
  constexpr int BLOCK = TPR < 256 ? 256 : TPR;
  const size_t smem = (size_t)staged_words(a.cols, SHIFT) * 4;
  if (NV * TPR * 8 > 4096) {
    static PerDeviceOnce once;
    int dev;
    if (once.need(&dev)) {
      const cudaError_t e = cudaFuncSetAttribute(layernorm_many_kernel<IO, NV, TPR, BLOCK, DROP, SHIFT, ROUND>,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024);
      if (e != cudaSuccess) return q8_code(e);
      once.mark(dev);
    }
  }
  const int sms = q8_sms();
  if (sms < 1) return PRM_ERR_CUDA;
  return q8_code(launch_after(layernorm_many_kernel<IO, NV, TPR, BLOCK, DROP, SHIFT, ROUND>,
                              (unsigned)(sms * layernorm_blocks(TPR, BLOCK)), BLOCK, smem, stream, 0, a));
}
template <typename IO, bool DROP, bool SHIFT, int NV, int TPR>
int launch_layernorm_many(const LayerNormArgs& a, cudaStream_t stream) {
  // 64 registers per thread leave no room for the step beside the generator (16384 x 2048 with dropout: 60 us, with it 13 more)
  if constexpr (!DROP || TPR >= 256) {
    if (a.rows_per_group >= a.rows) return launch_layernorm_many_as<IO, DROP, SHIFT, NV, TPR, true>(a, stream);
  }
  return launch_layernorm_many_as<IO, DROP, SHIFT, NV, TPR, false>(a, stream);
}
template <typename IO, bool DROP, bool SHIFT>
int run_layernorm(const LayerNormArgs& a, cudaStream_t stream) {
  const int64_t c = (int64_t)a.cols + (SHIFT ? 7 : 0);         // a row may need one more oct
  // At least some rows for each line of a block, of groups that are worth their weights' way to shared memory.
  const bool many = a.rows * a.cols >= (int64_t)148 * 4 * 4 * 4096 && a.rows_per_group >= 16;
#define PRM_TRY(NV, TPR)                                                                              \
  if (c <= 8 * NV * TPR) {                                                                            \
    if constexpr (sizeof(IO) == 2) {                                                                  \
      if (many) return launch_layernorm_many<IO, DROP, SHIFT, NV, TPR>(a, stream);                    \
    }                                                                                                 \
    return launch_layernorm<IO, DROP, SHIFT, NV, TPR>(a, stream);                                     \
  }
  PRM_TRY(1, 8)
  PRM_TRY(1, 16)
  PRM_TRY(1, 32)
  PRM_TRY(2, 32)
  PRM_TRY(2, 64)
  PRM_TRY(2, 128)
  PRM_TRY(2, 256)
  // half of the threads idle with the next size (8192 x 4097: 85 us, with it 19 more)
  if (c <= 8 * 3 * 256) return launch_layernorm<IO, DROP, SHIFT, 3, 256>(a, stream);
  PRM_TRY(2, 512)
#undef PRM_TRY
  if (c <= 8 * 2 * 1024) return launch_layernorm<IO, DROP, SHIFT, 2, 1024>(a, stream);
  return run_layernorm_single<IO>(a, stream);
}

}  // namespace
}  // namespace prm
