// Gradient of the layer norm at h, with xhat = (h - mean) rstd and g = grad_y w:
//
//   grad_r = rstd (g - mean(g) - xhat mean(g xhat)) + grad_h       (the residual's, and x's without dropout)
//   grad_x = grad_r dropped out like x
//   grad_w = sum over a group's rows of grad_y xhat,  grad_b = sum over a group's rows of grad_y
//
// Bound by HBM (8 bytes per element of a bf16 stream with grad_h, 10 with dropout).  Blocks walk the rows of
// one group; a thread keeps the same columns in all its rows, so that its share of grad_w and grad_b stays in
// registers, and the next row's loads are under way while this one is summed.  With several blocks to a group
// their lines of sums are added by a second launch, in a fixed order.  Measured: 8192 x 4096 in bf16 with grad_h 51 us, 5.2
// TB/s (fp32 85 us, 6.3), with dropout 78 us; 16384 x 2048 with a weight for each of 64 groups 50 us; 131072 x 128 29 us;
// 8192 x 4097 100 us; by single elements 4096 x 12288 364 us.
#include "layernorm.cuh"

namespace prm {
namespace {

struct LayerNormGradArgs {
  const void* gy;
  const void* h;
  const float* mean;
  const float* rstd;
  const void* gh;          // may be null
  void* gr;
  void* gx;                // dropout only
  void* gw;                // may be null
  void* gb;                // may be null
  float* part;             // [groups * parts][2][cols]
  int64_t ld_gy, ld_h, ld_gh, ld_gr, ld_gx, rows, rows_per_group;
  int cols, parts;
  Affine affine;           // bias unused
  Drop drop;
};

__device__ __forceinline__ void store_weight(void* out, int fp32, int64_t at, float v) {
  if (fp32) reinterpret_cast<float*>(out)[at] = v;
  else reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(v);
}

// Blocks per SM of the kernel below: 128 registers per thread with two octs or 32-bit elements (16384 x 2048 in fp32: 84 us,
// with 85 registers 35 more), else 85.
template <typename IO>
constexpr int layernorm_grad_blocks(int nv, int block) {
  return (nv == 1 && sizeof(IO) == 2 ? 768 : 512) / block;
}

template <typename IO, int NV, int TPR, int BLOCK, bool DROP, bool SHIFT>
__global__ void __launch_bounds__(BLOCK, layernorm_grad_blocks<IO>(NV, BLOCK)) layernorm_grad_kernel(const LayerNormGradArgs a) {
  constexpr int kRows = BLOCK / TPR, kWide = NV * TPR * 8;
  __shared__ float sums[kRows > 1 ? kRows : 1][kRows > 1 ? kWide : 1];
  __shared__ __align__(16) float red[2][kRows][TPR > 32 ? TPR / 32 * 2 : 1];
  grid_wait();
  grid_trigger();
  const int64_t group = blockIdx.x / (unsigned)a.parts, row0 = group * a.rows_per_group;
  const int part = (int)(blockIdx.x % (unsigned)a.parts), line = threadIdx.x / TPR;
  const int64_t step = (int64_t)a.parts * kRows, rows = a.rows_per_group;
  const int64_t first = (int64_t)part * kRows;
  // All rows of a thread start alike: `step` is a multiple of eight, or there is one row only.
  const int shift = SHIFT ? oct_shift(reinterpret_cast<const IO*>(a.h) + (row0 + first + line) * a.ld_h) : 0;
  const int c0 = (int)(threadIdx.x % TPR) * 8 - shift;
  const uint64_t number = DROP ? drop_number(a.drop) : 0;
  const float over = 1.f / (float)a.cols;
  float2 w[NV][4], gw[NV][4], gb[NV][4];
  Oct<IO> next[NV][3];
  float next_mean = 0.f, next_rstd = 0.f;
  // Asks the L2 for a row's lines, one lane for 128 bytes.  (8192 x 4096: 8 us less with it and the loop unrolled twice, so
  // that no registers are copied.  Rows that start anywhere spill and take 20 us more.)
  auto ask = [&](int64_t local) {
    if (local < rows && threadIdx.x % (16 / sizeof(IO)) == 0) {
      const int64_t row = row0 + local;
      const IO* gy = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
      const IO* h = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
      const IO* gh = reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * TPR * 8;
        if (c >= 0 && c < a.cols) {
          asm volatile("prefetch.global.L2 [%0];" ::"l"(gy + c));
          asm volatile("prefetch.global.L2 [%0];" ::"l"(h + c));
          if (a.gh) asm volatile("prefetch.global.L2 [%0];" ::"l"(gh + c));
        }
      }
    }
  };
  auto fetch = [&](int64_t local) {
    if (local < rows) {
      const int64_t row = row0 + local;
      next_mean = a.mean[row];
      next_rstd = a.rstd[row];
      if constexpr (SHIFT) {
        const OctRow<IO> gyr(a.gy, row, a.rows, a.ld_gy, a.cols), hr(a.h, row, a.rows, a.ld_h, a.cols);
        const OctRow<IO> ghr(a.gh ? a.gh : a.h, row, a.rows, a.gh ? a.ld_gh : a.ld_h, a.cols);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int c = c0 + v * TPR * 8;
          gyr.load(c, a.cols, next[v][0]);
          hr.load(c, a.cols, next[v][1]);
          if (a.gh) ghr.load(c, a.cols, next[v][2]);
        }
      } else {
        const IO* gy = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
        const IO* h = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
        const IO* gh = reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int c = c0 + v * TPR * 8;
          if (c < a.cols) {
            next[v][0].load_stream(gy + c);
            next[v][1].load_stream(h + c);
            if (a.gh) next[v][2].load_stream(gh + c);
          }
        }
      }
    }
  };
  fetch(first + line);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) gw[v][e] = gb[v][e] = make_float2(0.f, 0.f);
    affine_weight(a.affine, group, c0 + v * TPR * 8, a.cols, w[v]);
  }
  constexpr bool AHEAD = kRows == 1 && !SHIFT;
  if constexpr (AHEAD) ask(first + line + step);
  int turn = 0;
#pragma unroll (AHEAD ? 2 : 1)
  for (int64_t base = first; base < rows; base += step, turn ^= 1) {
    const int64_t local = base + line, row = row0 + local;
    const int cols = local < rows ? a.cols : 0;
    Oct<IO> now[NV][3];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int k = 0; k < 3; ++k) now[v][k] = next[v][k];
    // xhat is a product of the difference: with -mean rstd rounded by itself (one fused step), a mean of 10^5 deviations would put
    // each xhat of the row off by up to 0.004, a constant row's too.
    const float2 rs2 = make_float2(next_rstd, next_rstd), off2 = make_float2(-next_mean, -next_mean);
    fetch(local + step);
    if constexpr (AHEAD) ask(local + 2 * step);
    float2 sg2 = make_float2(0.f, 0.f), sx2 = sg2;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      if (c < cols) {
        float2 g[4], xhat[4];
        now[v][0].get(g);
        now[v][1].get(xhat);
        if constexpr (SHIFT) {
          clear_outside(c, cols, g);
          clear_outside(c, cols, xhat);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xhat[e] = mul2(add2(xhat[e], off2), rs2);
          gw[v][e] = fma2(g[e], xhat[e], gw[v][e]);
          gb[v][e] = add2(gb[v][e], g[e]);
          g[e] = mul2(g[e], w[v][e]);
          sg2 = add2(sg2, g[e]);
          sx2 = fma2(g[e], xhat[e], sx2);
        }
      }
    }
    float total[2] = {sg2.x + sg2.y, sx2.x + sx2.y};
    row_sums<TPR, BLOCK>(total, red[turn][line]);
    const float2 mg2 = make_float2(-total[0] * over, -total[0] * over), mx2 = make_float2(-total[1] * over * rs2.x, -total[1] * over * rs2.x);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * TPR * 8;
      if (c < cols) {
        float2 g[4], h[4], o[4];
        now[v][0].get(g);
        now[v][1].get(h);
        if (a.gh) {
          now[v][2].get(o);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fma2(fma2(add2(h[e], off2), mx2, fma2(g[e], w[v][e], mg2)), rs2, o[e]);
        IO* gr = reinterpret_cast<IO*>(a.gr) + row * a.ld_gr;
        if constexpr (SHIFT) {
          store_part(gr, c, cols, o);
        } else {
          Oct<IO> out;
          out.set(o);
          out.store(gr + c);
        }
        if constexpr (DROP) {
          IO* gx = reinterpret_cast<IO*>(a.gx) + row * a.ld_gx;
          drop_oct<!SHIFT>(a.drop, number, (uint32_t)row, c, o);
          if constexpr (SHIFT) {
            store_part(gx, c, cols, o);
          } else {
            Oct<IO> out;
            out.set(o);
            out.store(gx + c);
          }
        }
      }
    }
  }
  if (!a.gw && !a.gb) return;
  if (kRows == 1 && !SHIFT && a.parts > 1) {                     // the block's sums to its line of the scratch, as they are
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * TPR * 8;
        if (c < a.cols) {
          Oct<float> o;
          o.set(which ? gb[v] : gw[v]);
          o.store(a.part + ((int64_t)blockIdx.x * 2 + which) * a.cols + c);
        }
      }
    }
    return;
  }
  // The block's sums: to its line of the scratch, or, where it has the group to itself, to the gradients.
  auto put = [&](int which, int c, float v) {
    if (a.parts > 1) a.part[((int64_t)blockIdx.x * 2 + which) * a.cols + c] = v;
    else if (which ? a.gb : a.gw) store_weight(which ? a.gb : a.gw, a.affine.fp32, group * a.cols + c, v);
  };
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (kRows > 1) __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int c = c0 + v * TPR * 8 + k;
        const float2 s = which ? gb[v][k / 2] : gw[v][k / 2];
        if (c >= 0 && c < a.cols) {
          if constexpr (kRows > 1) sums[line][c] = k & 1 ? s.y : s.x;
          else put(which, c, k & 1 ? s.y : s.x);
        }
      }
    }
    if constexpr (kRows > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += BLOCK) {
        float s = 0.f;
#pragma unroll
        for (int l = 0; l < kRows; ++l) s += sums[l][c];
        put(which, c, s);
      }
    }
  }
}

// Any alignment, any length: two passes over the row, four elements per thread at a time; the block's share of
// the sums is collected in its line of the scratch (each thread its own columns).
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS) layernorm_grad_single_kernel(const LayerNormGradArgs a) {
  __shared__ __align__(16) float red[2][THREADS / 32 * 2];
  grid_wait();
  grid_trigger();
  const int64_t group = blockIdx.x / (unsigned)a.parts, row0 = group * a.rows_per_group;
  const int64_t first = blockIdx.x % (unsigned)a.parts;
  const uint64_t number = drop_number(a.drop);
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.cols;
  int turn = 0;
  for (int64_t local = first; local < a.rows_per_group; local += a.parts, turn ^= 1) {
    const int64_t row = row0 + local;
    const IO* gyp = reinterpret_cast<const IO*>(a.gy) + row * a.ld_gy;
    const IO* hp = reinterpret_cast<const IO*>(a.h) + row * a.ld_h;
    const IO* ghp = a.gh ? reinterpret_cast<const IO*>(a.gh) + row * a.ld_gh : nullptr;
    IO* grp = reinterpret_cast<IO*>(a.gr) + row * a.ld_gr;
    IO* gxp = a.drop.threshold ? reinterpret_cast<IO*>(a.gx) + row * a.ld_gx : nullptr;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sg = 0.f, sx = 0.f;
    for (int c = threadIdx.x * 4; c < a.cols; c += THREADS * 4) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c + k < a.cols) {
          const float gy = to_f32(gyp[c + k]), xhat = (to_f32(hp[c + k]) - mean) * rstd;
          const float g = gy * affine_weight1(a.affine, group, c + k);
          sg += g;
          sx += g * xhat;
          part[c + k] = (local == first ? 0.f : part[c + k]) + gy * xhat;
          part[a.cols + c + k] = (local == first ? 0.f : part[a.cols + c + k]) + gy;
        }
      }
    }
    float total[2] = {sg, sx};
    row_sums<THREADS, THREADS>(total, red[turn]);
    const float mg = total[0] / (float)a.cols, mx = total[1] / (float)a.cols;
    for (int c = threadIdx.x * 4; c < a.cols; c += THREADS * 4) {
      uint4 w = make_uint4(~0u, ~0u, ~0u, ~0u);
      if (gxp) w = drop_words(a.drop, number, (uint32_t)row, (uint32_t)c >> 2);
      const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c + k < a.cols) {
          const float gy = to_f32(gyp[c + k]), xhat = (to_f32(hp[c + k]) - mean) * rstd;
          float o = rstd * (gy * affine_weight1(a.affine, group, c + k) - mg - xhat * mx);
          if (ghp) o += to_f32(ghp[c + k]);
          from_f32(grp + c + k, o);
          if (gxp) from_f32(gxp + c + k, dropped(a.drop, word[k], o));
        }
      }
    }
  }
}

// The blocks' lines added, all in a fixed order.  Many lines: 32 columns of one of the two gradients of a group per block, a line
// per warp at a time, so that all are under way together.
__global__ void __launch_bounds__(1024) layernorm_grad_sum_kernel(const LayerNormGradArgs a, int chunks) {
  __shared__ float s[32][33];
  grid_wait();
  grid_trigger();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int which = blockIdx.x & 1;
  const int64_t group = (blockIdx.x >> 1) / (unsigned)chunks;
  const int64_t c = (int64_t)((blockIdx.x >> 1) % (unsigned)chunks) * 32 + lane;
  void* out = which ? a.gb : a.gw;
  if (!out) return;
  float sum = 0.f;
  if (c < a.cols) {
    const float* p = a.part + (group * a.parts * 2 + which) * a.cols + c;
#pragma unroll 10
    for (int l = warp; l < a.parts; l += 32) sum += __ldcg(p + (int64_t)l * 2 * a.cols);
  }
  s[warp][lane] = sum;
  __syncthreads();
  const float v = warp_sum(s[lane][warp]);                       // of column `warp`
  const int64_t at = c - lane + warp;
  if (lane == 0 && at < a.cols) store_weight(out, a.affine.fp32, group * a.cols + at, v);
}
// Few lines (of many groups): a thread per column.
__global__ void __launch_bounds__(256) layernorm_grad_sum_few_kernel(const LayerNormGradArgs a, int chunks) {
  grid_wait();
  grid_trigger();
  const int which = blockIdx.x & 1;
  const int64_t group = (blockIdx.x >> 1) / (unsigned)chunks;
  const int64_t c = (int64_t)((blockIdx.x >> 1) % (unsigned)chunks) * 256 + threadIdx.x;
  void* out = which ? a.gb : a.gw;
  if (!out || c >= a.cols) return;
  const float* p = a.part + (group * a.parts * 2 + which) * a.cols + c;
  float sum = 0.f;
#pragma unroll 8
  for (int l = 0; l < a.parts; ++l) sum += __ldcg(p + (int64_t)l * 2 * a.cols);
  store_weight(out, a.affine.fp32, group * a.cols + c, sum);
}

int launch_sum(const LayerNormGradArgs& a, int64_t groups, cudaStream_t stream) {
  if (!a.gw && !a.gb) return PRM_OK;
  if (a.parts > kLinesPerThread) {
    const int chunks = (a.cols + 31) / 32;
    return q8_code(launch_after(layernorm_grad_sum_kernel, (unsigned)(groups * chunks * 2), 1024, 0, stream, 0, a, chunks));
  }
  const int chunks = (a.cols + 255) / 256;
  return q8_code(launch_after(layernorm_grad_sum_few_kernel, (unsigned)(groups * chunks * 2), 256, 0, stream, 0, a, chunks));
}

template <typename IO>
int launch_layernorm_grad_single(LayerNormGradArgs a, int64_t groups, cudaStream_t stream) {
  a.parts = (int)layernorm_parts(a.rows_per_group, groups, a.cols, 1, 444, false);
  const int code = a.cols <= 1024
                       ? q8_code(launch_after(layernorm_grad_single_kernel<IO, 256>, (unsigned)(groups * a.parts), 256, 0,
                                              stream, 0, a))
                       : q8_code(launch_after(layernorm_grad_single_kernel<IO, 1024>, (unsigned)(groups * a.parts), 1024, 0,
                                              stream, 0, a));
  return code == PRM_OK ? launch_sum(a, groups, stream) : code;
}
template <typename IO, bool DROP, bool SHIFT, int NV, int TPR, int BLOCK>
int launch_layernorm_grad(LayerNormGradArgs a, int64_t groups, cudaStream_t stream) {
  const int blocks = 148 * layernorm_grad_blocks<IO>(NV, BLOCK);
  a.parts = (int)layernorm_parts(a.rows_per_group, groups, a.cols, BLOCK / TPR, blocks, SHIFT);
  if (SHIFT && a.parts > layernorm_lines(a.rows_per_group, groups, a.cols)) {
    if (a.ld_h % 8 != 0) return launch_layernorm_grad_single<IO>(a, groups, stream);
    a.parts = (int)layernorm_parts(a.rows_per_group, groups, a.cols, BLOCK / TPR, blocks, false);       // all rows start alike
  }
  const int code = q8_code(launch_after(layernorm_grad_kernel<IO, NV, TPR, BLOCK, DROP, SHIFT>, (unsigned)(groups * a.parts),
                                        BLOCK, 0, stream, 0, a));
  return code == PRM_OK && a.parts > 1 ? launch_sum(a, groups, stream) : code;
}

template <typename IO, bool DROP, bool SHIFT>
int run_layernorm_grad(const LayerNormGradArgs& a, int64_t groups, cudaStream_t stream) {
  const int64_t c = (int64_t)a.cols + (SHIFT ? 7 : 0);
  // Two octs per thread halve what a row's reduction costs each; of 32-bit elements they leave the registers, but a block of
  // 1024 threads has too few for one (4096 x 8192 in fp32: 158 us, so 60 more).
  constexpr int NV = sizeof(IO) == 2 ? 2 : 1, T = NV == 2 ? 1 : 2;
  if (c <= 64) return launch_layernorm_grad<IO, DROP, SHIFT, 1, 8, 256>(a, groups, stream);
  if (c <= 128) return launch_layernorm_grad<IO, DROP, SHIFT, 1, 16, 256>(a, groups, stream);
  if (c <= 256) return launch_layernorm_grad<IO, DROP, SHIFT, 1, 32, 256>(a, groups, stream);
  if (c <= 512) return launch_layernorm_grad<IO, DROP, SHIFT, NV, 32 * T, 128>(a, groups, stream);
  if (c <= 1024) return launch_layernorm_grad<IO, DROP, SHIFT, NV, 64 * T, 64 * T>(a, groups, stream);
  if (c <= 2048) return launch_layernorm_grad<IO, DROP, SHIFT, NV, 128 * T, 128 * T>(a, groups, stream);
  if (c <= 4096) return launch_layernorm_grad<IO, DROP, SHIFT, NV, 256 * T, 256 * T>(a, groups, stream);
  if (c <= 8192) return launch_layernorm_grad<IO, DROP, SHIFT, 2, 512, 512>(a, groups, stream);
  return launch_layernorm_grad_single<IO>(a, groups, stream);
}
template <typename IO>
int run_any(const LayerNormGradArgs& a, int64_t groups, cudaStream_t stream) {
  const bool drop = a.drop.threshold != 0;
  const bool octs = a.cols % 8 == 0 && a.ld_gy % 8 == 0 && a.ld_h % 8 == 0 && a.ld_gr % 8 == 0 && aligned16(a.gy) &&
                    aligned16(a.h) && aligned16(a.gr) && (!a.gh || (a.ld_gh % 8 == 0 && aligned16(a.gh))) &&
                    (!drop || (a.ld_gx % 8 == 0 && aligned16(a.gx)));
  if (octs)
    return drop ? run_layernorm_grad<IO, true, false>(a, groups, stream) : run_layernorm_grad<IO, false, false>(a, groups, stream);
  if (octs_alike<IO>(a.h, a.ld_h, a.gy, a.ld_gy) && octs_alike<IO>(a.h, a.ld_h, a.gr, a.ld_gr) &&
      (!a.gh || octs_alike<IO>(a.h, a.ld_h, a.gh, a.ld_gh)) && (!drop || octs_alike<IO>(a.h, a.ld_h, a.gx, a.ld_gx)))
    return drop ? run_layernorm_grad<IO, true, true>(a, groups, stream) : run_layernorm_grad<IO, false, true>(a, groups, stream);
  return launch_layernorm_grad_single<IO>(a, groups, stream);
}

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" size_t prm_layernorm_scratch_bytes(int64_t rows, int64_t cols, int64_t rows_per_group) {
  if (rows < 1 || cols < 1 || rows_per_group < 1) return 0;
  rows_per_group = std::min(rows_per_group, rows);
  const int64_t groups = rows / rows_per_group;
  return (size_t)(groups * layernorm_lines(rows_per_group, groups, cols)) * 2 * (size_t)cols * 4;
}

extern "C" int prm_layernorm_backward(const void* grad_y, int64_t ld_grad_y, const void* h, int64_t ld_h, const float* mean,
                                      const float* rstd, const void* weight, int64_t ld_weight, const void* grad_h,
                                      int64_t ld_grad_h, int64_t rows, int64_t cols, int64_t rows_per_group, int io_fp32,
                                      int weight_fp32, int add_one, double p, uint64_t seed, uint64_t offset,
                                      const uint64_t* counter, void* grad_residual, int64_t ld_grad_residual, void* grad_x,
                                      int64_t ld_grad_x, void* grad_weight, void* grad_bias, void* scratch,
                                      size_t scratch_bytes, void* cuda_stream) {
  if (rows < 0 || rows_per_group < 1 || !drop_ok(p)) return PRM_ERR_ARG;
  if (cols < 1 || cols > 0x7fffffffLL - 8192 || rows > 0x7fffffffLL) return PRM_ERR_SHAPE;
  const Drop drop = make_drop(p, seed, offset, counter);
  if (!layernorm_ld_ok(ld_grad_y) || !layernorm_ld_ok(ld_h) || (weight && !layernorm_ld_ok(ld_weight)) ||
      (grad_h && !layernorm_ld_ok(ld_grad_h)) || ld_grad_residual < cols || !layernorm_ld_ok(ld_grad_residual) ||
      (drop.threshold && (ld_grad_x < cols || !layernorm_ld_ok(ld_grad_x))))
    return PRM_ERR_SHAPE;
  const int ws = weight_fp32 ? 4 : 2;
  if (((uintptr_t)grad_weight | (uintptr_t)grad_bias) % ws != 0) return PRM_ERR_ALIGN;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (rows == 0) {                        // empty sums, of one group
    cudaError_t e = grad_weight ? cudaMemsetAsync(grad_weight, 0, (size_t)cols * ws, stream) : cudaSuccess;
    if (e == cudaSuccess && grad_bias) e = cudaMemsetAsync(grad_bias, 0, (size_t)cols * ws, stream);
    return q8_code(e);
  }
  rows_per_group = std::min(rows_per_group, rows);
  const int64_t groups = rows / rows_per_group;
  if (groups * rows_per_group != rows || !layernorm_grids_ok(rows_per_group, groups, cols)) return PRM_ERR_SHAPE;
  if (!grad_y || !h || !mean || !rstd || !grad_residual || (drop.threshold && !grad_x) || !scratch) return PRM_ERR_ARG;
  if (scratch_bytes < prm_layernorm_scratch_bytes(rows, cols, rows_per_group)) return PRM_ERR_WORKSPACE;
  const uintptr_t stream_bits = (uintptr_t)grad_y | (uintptr_t)h | (uintptr_t)grad_h | (uintptr_t)grad_residual |
                                (uintptr_t)(drop.threshold ? grad_x : nullptr);
  if (stream_bits % (io_fp32 ? 4 : 2) != 0 || (uintptr_t)weight % ws != 0 || ((uintptr_t)mean | (uintptr_t)rstd) % 4 != 0 ||
      ((uintptr_t)scratch & 15) != 0 || (uintptr_t)counter % 8 != 0)
    return PRM_ERR_ALIGN;
  const LayerNormGradArgs a = {grad_y, h, mean, rstd, grad_h, grad_residual, grad_x, grad_weight, grad_bias, (float*)scratch,
                               ld_grad_y, ld_h, ld_grad_h, ld_grad_residual, ld_grad_x, rows, rows_per_group,
                               (int)cols, 1, {weight, nullptr, ld_weight, 0, weight_fp32, add_one}, drop};
  return io_fp32 ? run_any<float>(a, groups, stream) : run_any<__nv_bfloat16>(a, groups, stream);
}
