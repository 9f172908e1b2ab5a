// The quantiser: a matrix to 8-bit codes with one scale per row, per column, or both ways at once.
//
//   by rows:     t = x * fold_cols,   scale[i] = max_j |t_ij| / limit,   code = round(t * limit / max)
//   by columns:  t = x * fold_rows,   scale[j] = max_i |t_ij| / limit,   likewise
//
// The folds carry the scales that run along the sum of the product that will read the codes: a
// product can take out one factor per row of its left operand and per column of its right one, and
// nothing that varies inside its sums.
//
// Three numbers per element (read, two writes at most) make this HBM's work, but a column's scale
// waits for the whole column.  The streaming kernel reads the matrix once, writes the codes by row on
// the way and keeps the largest magnitude of every column; after a grid-wide reduction of these it
// goes over the rows again in the opposite order, the last ones still in shared memory, those before
// them in L2.
#include <cooperative_groups.h>

#include "row_ring.cuh"
#include "tcgen05.cuh"

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
  float* part;              // [blocks][panel] the same of a block's rows
  int64_t rows, ld_x, ld_qr, ld_qc;
  int cols, format;
  int panel, panels;        // columns that a block of the streaming kernel works on; cols / panel
  float minus_zero = -0.f;  // see int8_bits
};

// x * f for one oct (f: eight factors from c on, or null; 16-byte loads where they are aligned).
__device__ __forceinline__ void fold_oct(const float* f, int c, float2 (&t)[4]) {
  if (!f) return;
  float2 m[4];
  if (((uintptr_t)f & 15) == 0) {
    Oct<float> o;
    o.load(f + c);
    o.get(m);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = make_float2(__ldg(f + c + 2 * e), __ldg(f + c + 2 * e + 1));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = mul2(t[e], m[e]);
}

// One row per group of TPR threads, in registers between the maximum and the rounding.
template <typename IO, int NV, int TPR>
__global__ void __launch_bounds__(TPR <= 32 ? 256 : TPR) quantize_rows_kernel(const QuantArgs a) {
  constexpr int kRows = TPR <= 32 ? 256 / TPR : 1;
  __shared__ float red[64];
  grid_wait();
  grid_trigger();
  const int c0 = (threadIdx.x % TPR) * 8;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  const int cols = row < a.rows ? a.cols : 0;                   // what this thread has of the row's columns
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  Oct<IO> xv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (c0 + v * TPR * 8 < cols) xv[v].load_stream(x + c0 + v * TPR * 8);
  float2 t[NV][4];
  float none = 0.f, top = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * TPR * 8;
    if (c < cols) {
      xv[v].get(t[v]);
      fold_oct(a.fold_cols, c, t[v]);
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max_abs(top, t[v][e]);
    }
  }
  block_sum_top<TPR>(none, top, red);
  store_octs<NV>(a.q_rows + row * a.ld_qr, t, c0, TPR * 8, cols, top, a.format, a.minus_zero);
  if (c0 == 0 && cols) a.scale_rows[row] = q8_scale(top, q8_limit(a.format));
}

// Rows that start anywhere (odd widths), or too wide for the kernel above: the same on octs aligned in
// memory.
template <typename IO, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) quantize_rows_shifted_kernel(const QuantArgs a) {
  constexpr int kRows = TPR == 32 ? 8 : 1;
  __shared__ float red[64];
  __shared__ uint64_t stage[kRows][NV * TPR + 1];
  grid_wait();
  grid_trigger();
  const int o0 = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (row >= a.rows) return;
  const OctRow<IO> x(a.x, row, a.rows, a.ld_x, a.cols);
  const int shift = oct_shift(x.p);
  Oct<IO> xv[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) x.load((o0 + v * TPR) * 8 - shift, a.cols, xv[v]);
  float2 t[NV][4];
  float none = 0.f, top = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (o0 + v * TPR) * 8 - shift;
    get_part(xv[v], c, a.cols, t[v]);
    if (a.fold_cols) {
      float2 f[4];
      load_factors(a.fold_cols, 1, c, a.cols, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[v][e] = mul2(t[v][e], f[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max_abs(top, t[v][e]);
  }
  block_sum_top<TPR>(none, top, red);
  store_octs_shifted<NV, TPR>(stage[threadIdx.x / TPR], a.q_rows + row * a.ld_qr, t, o0, shift, a.cols, top, a.format, a.minus_zero);
  if (o0 == 0) a.scale_rows[row] = q8_scale(top, q8_limit(a.format));
}

// Any alignment, any length: two passes over the row.
template <typename IO, int THREADS>
__global__ void __launch_bounds__(THREADS) quantize_rows_single_kernel(const QuantArgs a) {
  __shared__ float red[64];
  grid_wait();
  grid_trigger();
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
  const bool finite = q8_finite(top);
  const float mul = q8_mul(top, q8_limit(a.format));
#pragma unroll 4
  for (int c = threadIdx.x; c < a.cols; c += THREADS)
    a.q_rows[row * a.ld_qr + c] = finite ? code1(value(c), mul, a.format) : 0;
  if (threadIdx.x == 0) a.scale_rows[row] = q8_scale(top, q8_limit(a.format));
}

// Largest magnitude of every column, any alignment: a block takes 256 columns of a slab of rows; the
// maximum of the bit patterns (NaN above infinity above numbers) joins the slabs in any order alike.
constexpr int kColThreads = 256;
template <typename IO>
__global__ void __launch_bounds__(kColThreads) column_top_kernel(const QuantArgs a, int slab) {
  const int c = blockIdx.x * kColThreads + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * slab, r1 = min(a.rows, r0 + slab);
  float top = 0.f;
  const IO* x = reinterpret_cast<const IO*>(a.x) + r0 * a.ld_x + c;
#pragma unroll 8
  for (int64_t r = r0; r < r1; ++r, x += a.ld_x)
    top = max_abs(top, make_float2(__fmul_rn(to_f32(*x), a.fold_rows ? __ldg(a.fold_rows + r) : 1.f), 0.f));
  atomicMax(a.top + c, __float_as_uint(top));
}

// Eight codes, a factor for each.
template <int FORMAT>
__device__ __forceinline__ uint2 column_codes(const float2 (&t)[4], const float2 (&mul)[4], float nz) {
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float2 a = t[2 * k], b = t[2 * k + 1], f = mul[2 * k], g = mul[2 * k + 1];
    if constexpr (FORMAT == PRM_Q8_INT8) {
      const float2 x = int8_bits(a, f, nz), y = int8_bits(b, g, nz);
      w[k] = __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040),
                         __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
    } else {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(mul2(a, f), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(mul2(b, g), __NV_SATFINITE, __NV_E4M3);
      w[k] = lo | (hi << 16);
    }
  }
  return make_uint2(w[0], w[1]);
}

template <typename IO>
__global__ void __launch_bounds__(kColThreads) quantize_cols_kernel(const QuantArgs a, int slab) {
  const int c = blockIdx.x * kColThreads + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * slab, r1 = min(a.rows, r0 + slab);
  const float top = __uint_as_float(a.top[c]), mul = q8_mul(top, q8_limit(a.format));
  const bool finite = q8_finite(top);
  if (blockIdx.y == 0) a.scale_cols[c] = q8_scale(top, q8_limit(a.format));
  const IO* x = reinterpret_cast<const IO*>(a.x) + r0 * a.ld_x + c;
  uint8_t* q = a.q_cols + r0 * a.ld_qc + c;
#pragma unroll 8
  for (int64_t r = r0; r < r1; ++r, x += a.ld_x, q += a.ld_qc)
    *q = finite ? code1(__fmul_rn(to_f32(*x), a.fold_rows ? __ldg(a.fold_rows + r) : 1.f), mul, a.format) : 0;
}

// A thread's share of one row of codes by column.
template <typename IO, int NV, int FORMAT>
__device__ __forceinline__ void back_row(uint8_t* q, const Oct<IO> (&x)[NV], const float2 (&mul)[NV][4], float fr,
                                         bool odd, int c0, int step, int cols, float nz) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * step;
    if (c < cols) {
      float2 t[4];
      x[v].get(t);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = mul2(t[e], make_float2(fr, fr));
      if (!odd) {
        *reinterpret_cast<uint2*>(q + c) = column_codes<FORMAT>(t, mul[v], nz);
      } else {
        float2 m[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[e] = mul[v][e];
          if (isnan(m[e].x)) t[e].x = m[e].x = 0.f;
          if (isnan(m[e].y)) t[e].y = m[e].y = 0.f;
        }
        *reinterpret_cast<uint2*>(q + c) = column_codes<FORMAT>(t, m, nz);
      }
    }
  }
}

// Codes by column: a cluster of up to eight blocks to a panel of LANES octs of columns, so that a column's
// scale waits for these and not for the grid.  A thread has one oct of one row in (blocks * kRowLanes); the
// rows of its last turn stay in its registers, those before them it finds in the L2.
constexpr int kPanelThreads = 256, kPanelCluster = 8, kPanelRows = 8;
template <typename IO, int LANES>
__global__ void __launch_bounds__(kPanelThreads) quantize_panel_kernel(const QuantArgs a) {
  constexpr int kRowLanes = kPanelThreads / LANES, kWidth = LANES * 8, kWarps = kPanelThreads / 32;
  static_assert(LANES <= 32 && kWidth <= kPanelThreads, "a warp holds whole rows of the panel, a thread has one column");
  __shared__ __align__(16) uint32_t own[kWarps][kWidth], all[kPanelCluster][kWidth];
  __shared__ __align__(16) float factor[kWidth];
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  grid_wait();
  grid_trigger();
  const uint32_t rank = cluster_ctarank(), blocks = cluster_nctarank();
  const int cbase = (int)(blockIdx.x / blocks) * kWidth, lane = threadIdx.x % LANES;
  const int cols = a.cols - cbase < lane * 8 ? 0 : a.cols - cbase - lane * 8;   // from this thread's oct on
  const int64_t first = (int64_t)rank * kRowLanes + threadIdx.x / LANES, step = blocks * kRowLanes;
  const IO* x = reinterpret_cast<const IO*>(a.x) + cbase + lane * 8;
  uint8_t* q = a.q_cols + cbase + lane * 8;
  const int64_t turns = (a.rows + step * kPanelRows - 1) / (step * kPanelRows);
  Oct<IO> v[kPanelRows];
  float f[kPanelRows];
  auto fetch = [&](int64_t turn) {
#pragma unroll
    for (int k = 0; k < kPanelRows; ++k) {
      const int64_t r = first + (turn * kPanelRows + k) * step;
      v[k].zero();
      f[k] = 1.f;
      if (r < a.rows && cols > 0) {
        v[k].load(x + r * a.ld_x);
        if (a.fold_rows) f[k] = __ldg(a.fold_rows + r);
      }
    }
  };
  float top[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) top[e] = 0.f;
  for (int64_t turn = 0; turn < turns; ++turn) {
    fetch(turn);
#pragma unroll
    for (int k = 0; k < kPanelRows; k += 2) {
      float2 t[4], u[4];
      v[k].get(t);
      v[k + 1].get(u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        t[e] = mul2(t[e], make_float2(f[k], f[k]));
        u[e] = mul2(u[e], make_float2(f[k + 1], f[k + 1]));
        top[2 * e] = max_abs(top[2 * e], make_float2(t[e].x, u[e].x));
        top[2 * e + 1] = max_abs(top[2 * e + 1], make_float2(t[e].y, u[e].y));
      }
    }
  }
  // Joined as bit patterns (NaN above infinity above numbers): over the warp's rows, the block's warps, the
  // cluster's blocks.
  uint32_t bits[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bits[e] = __float_as_uint(top[e]);
#pragma unroll
    for (int o = LANES; o < 32; o *= 2) bits[e] = max(bits[e], __shfl_xor_sync(0xffffffffu, bits[e], o));
  }
  if (threadIdx.x % 32 < LANES) {
    uint4* to = reinterpret_cast<uint4*>(&own[threadIdx.x / 32][lane * 8]);
    to[0] = make_uint4(bits[0], bits[1], bits[2], bits[3]);
    to[1] = make_uint4(bits[4], bits[5], bits[6], bits[7]);
  }
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // all blocks of the cluster are there
  if (threadIdx.x < kWidth) {
    uint32_t most = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) most = max(most, own[w][threadIdx.x]);
    const uint32_t mine = smem_u32(&all[rank][threadIdx.x]);
#pragma unroll
    for (uint32_t r = 0; r < kPanelCluster; ++r)
      if (r < blocks) st_cluster_u32(cluster_map(mine, r), most);
  }
  cluster_barrier();
  bool odd = false;
  if (threadIdx.x < kWidth) {
    uint32_t most = 0;
#pragma unroll
    for (uint32_t r = 0; r < kPanelCluster; ++r)
      if (r < blocks) most = max(most, all[r][threadIdx.x]);
    const float t = __uint_as_float(most), limit = q8_limit(a.format);
    odd = !q8_finite(t);
    factor[threadIdx.x] = odd ? __uint_as_float(0x7fffffffu) : q8_mul(t, limit);
    if (rank == 0 && cbase + (int)threadIdx.x < a.cols) a.scale_cols[cbase + threadIdx.x] = q8_scale(t, limit);
  }
  odd = __syncthreads_or(odd);
  float2 mul[1][4];
  {
    Oct<float> o;
    o.load(factor + lane * 8);
    o.get(mul[0]);
  }
  for (int64_t turn = turns - 1;; --turn) {
#pragma unroll
    for (int k = 0; k < kPanelRows; ++k) {
      const int64_t r = first + (turn * kPanelRows + k) * step;
      if (r < a.rows) {
        const Oct<IO> one[1] = {v[k]};
        if (a.format == PRM_Q8_INT8) back_row<IO, 1, PRM_Q8_INT8>(q + r * a.ld_qc, one, mul, f[k], odd, 0, 0, cols, a.minus_zero);
        else back_row<IO, 1, PRM_Q8_E4M3>(q + r * a.ld_qc, one, mul, f[k], odd, 0, 0, cols, a.minus_zero);
      }
    }
    if (turn == 0) break;
    fetch(turn - 1);
  }
}

// Bytes of the matrix that the first walk leaves in the L2 for the second.
constexpr int64_t kKeep = (int64_t)64 << 20;

// The streaming kernel.  Blocks with the same blockIdx % panels work on the same panel of columns;
// with codes by row there is one panel, the whole width.  Phase 1: groups of W warps walk over sets of
// R rows, NV octs per thread and row.  Then the blocks' column maxima are joined (shared memory, scratch,
// a slice of the columns per block) between two grid-wide barriers of the cooperative launch.  Phase 2
// walks back.
template <typename IO, int W, int NV, int R, bool ROWS>
__global__ void __launch_bounds__(kRingThreads, 1) quantize_stream_kernel(const QuantArgs a, int stages, int* status) {
  constexpr int kStep = W * 32 * 8;
  __shared__ float slice[kRingThreads / 32][128];
  const int pan = blockIdx.x % a.panels, line = blockIdx.x / a.panels;
  const int lines = ((int)gridDim.x - pan + a.panels - 1) / a.panels;   // blocks of this panel
  const int cbase = pan * a.panel, cols = min(a.panel, a.cols - cbase);
  const int c0 = (threadIdx.x % (W * 32)) * 8;
  const void* const src[1] = {reinterpret_cast<const IO*>(a.x) + cbase};
  const int64_t ld[1] = {a.ld_x};
  RowRing<IO, W, R, 1> ring(ring_block<W, R>(), src, ld, a.rows, cols, stages, status);
  ring.place(line, lines);
  float* tops = reinterpret_cast<float*>(ring_memory() + (size_t)(kRingWarps / W) * stages * R * ring.row_bytes);
  // The column factors come from shared memory: eight neighbouring fp32 per thread and row are loads
  // of 32 sectors each (4096 x 8192 both ways with folds: 76 us).
  float* fold = tops + a.panel;
  if constexpr (ROWS) {
    if (a.fold_cols)
      for (int c = threadIdx.x; c < cols; c += kRingThreads) fold[c] = __ldg(a.fold_cols + c);
  }
  ring.start();
  float ct[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) ct[v][e] = 0.f;
  const int n = ring.producer ? 0 : ring.n;
  // What the second walk reads first stays in the L2: the rows that are read last, up to kKeep bytes in
  // all CTAs' rings together.
  if (ring.producer) {
    const int64_t set = (int64_t)R * (kRingWarps / W) * gridDim.x * ring.row_bytes;
    ring.serve(ring.n - stages - (int)(kKeep / set));
  }
  // The row factors are fetched a set ahead.
  auto row_factors = [&](int i, float (&f)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      f[r] = a.fold_rows && i >= 0 && i < n && r < ring.height(i) ? __ldg(a.fold_rows + ring.row(i) + r) : 1.f;
  };
  float next[R];
  row_factors(0, next);
  for (int i = 0; i < n; ++i) {
    const int64_t row = ring.row(i);
    const int h = ring.height(i);
    float fr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) fr[r] = next[r];
    row_factors(i + 1, next);
    float2 t[R][NV][4];
    float none[R], top[R];
#pragma unroll
    for (int r = 0; r < R; ++r) none[r] = top[r] = 0.f;
    if (ring.wait()) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * kStep;
        if (c < cols) {
          float2 f[R][4];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            Oct<IO> x;
            if (r < h) x.load(ring.at(r, 0) + c);
            else x.zero();
            x.get(t[r][v]);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[r][e] = mul2(t[r][v][e], make_float2(fr[r], fr[r]));
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ct[v][2 * e] = max_abs(ct[v][2 * e], make_float2(f[0][e].x, f[R - 1][e].x));
            ct[v][2 * e + 1] = max_abs(ct[v][2 * e + 1], make_float2(f[0][e].y, f[R - 1][e].y));
          }
          if constexpr (ROWS) {
            if (a.fold_cols) {
              float2 fc[4];
              Oct<float> o;
              o.load(fold + c);
              o.get(fc);
#pragma unroll
              for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) t[r][v][e] = mul2(t[r][v][e], fc[e]);
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e) top[r] = max_abs(top[r], t[r][v][e]);
          }
        }
      }
    }
    ring.release();
    ring.advance();
    if constexpr (ROWS) {
      ring.template reduce<false>(i, none, top);
      if (ring.ok) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r < h) {
            store_octs<NV>(a.q_rows + (row + r) * a.ld_qr, t[r], c0, kStep, cols, top[r], a.format, a.minus_zero);
            if (c0 == 0) a.scale_rows[row + r] = q8_scale(top[r], q8_limit(a.format));
          }
        }
      }
    }
  }
  cooperative_groups::grid_group grid = cooperative_groups::this_grid();
  grid_trigger();
  for (int g = 0; g < kRingWarps / W; ++g) {          // the groups take turns
    if (!ring.producer && ring.group == g) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * kStep;
        if (c < cols) {
          Oct<float> o;
          if (g > 0) {
            float2 m[4];
            o.load(tops + c);
            o.get(m);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              ct[v][2 * e] = max_abs(ct[v][2 * e], make_float2(m[e].x, 0.f));
              ct[v][2 * e + 1] = max_abs(ct[v][2 * e + 1], make_float2(m[e].y, 0.f));
            }
          }
          o.a = make_float4(ct[v][0], ct[v][1], ct[v][2], ct[v][3]);
          o.b = make_float4(ct[v][4], ct[v][5], ct[v][6], ct[v][7]);
          o.store(tops + c);
        }
      }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < cols; c += kRingThreads) a.part[(int64_t)blockIdx.x * a.panel + c] = tops[c];
  grid.sync();
  // this block's slice of the panel's columns: 128 at a time, four per lane, the lines dealt out to
  // the warps
  const int per = ((cols + lines - 1) / lines + 31) / 32 * 32, end = min(cols, (line + 1) * per);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int s0 = line * per; s0 < end; s0 += 128) {
    float m[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int l = warp; l < lines; l += kRingThreads / 32) {
      const float* p = a.part + (int64_t)(l * a.panels + pan) * a.panel + s0 + lane;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (s0 + k * 32 + lane < end) m[k] = max_abs(m[k], make_float2(__ldcg(p + k * 32), 0.f));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) slice[warp][k * 32 + lane] = m[k];
    __syncthreads();
    const int c = s0 + threadIdx.x;
    if (threadIdx.x < 128 && c < end) {
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < kRingThreads / 32; ++k) top = max_abs(top, make_float2(slice[k][threadIdx.x], 0.f));
      // a column without a number for a scale passes on a NaN, and gets zero codes
      reinterpret_cast<float*>(a.top)[cbase + c] = q8_finite(top) ? q8_mul(top, q8_limit(a.format)) : top - top;
      a.scale_cols[cbase + c] = q8_scale(top, q8_limit(a.format));
    }
    __syncthreads();
  }
  grid.sync();
  // All factors of this thread's columns are fetched before the first is used, in 16-byte pieces: one
  // load after the other from lines that every SM wants at once took 15 us.
  float2 mul[NV][4];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * kStep;
    if (c < cols) {
      const float4 p = __ldcg(reinterpret_cast<const float4*>(a.top + cbase + c));
      const float4 q = __ldcg(reinterpret_cast<const float4*>(a.top + cbase + c + 4));
      mul[v][0] = make_float2(p.x, p.y);
      mul[v][1] = make_float2(p.z, p.w);
      mul[v][2] = make_float2(q.x, q.y);
      mul[v][3] = make_float2(q.z, q.w);
    }
  }
  bool odd = false;                       // a column without a number for a scale among them
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (c0 + v * kStep < cols) {
#pragma unroll
      for (int e = 0; e < 4; ++e) odd = odd || isnan(mul[v][e].x) || isnan(mul[v][e].y);
    }
  ring.turn_back();
  if (ring.producer) ring.serve_back();
  row_factors(n - 1, next);
  for (int i = n - 1; i >= 0; --i) {
    const int64_t row = ring.row(i);
    const int h = ring.height(i);
    float fr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) fr[r] = next[r];
    row_factors(i - 1, next);
    Oct<IO> x[R][NV];
    if (ring.wait_back(i)) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < NV; ++v)
          if (r < h && c0 + v * kStep < cols) x[r][v].load(ring.at(r, 0) + c0 + v * kStep);
    }
    ring.release();
    ring.retreat();
    if (!ring.ok) continue;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r < h) {
        uint8_t* q = a.q_cols + (row + r) * a.ld_qc + cbase;
        if (a.format == PRM_Q8_INT8) back_row<IO, NV, PRM_Q8_INT8>(q, x[r], mul, fr[r], odd, c0, kStep, cols, a.minus_zero);
        else back_row<IO, NV, PRM_Q8_E4M3>(q, x[r], mul, fr[r], odd, c0, kStep, cols, a.minus_zero);
      }
    }
  }
  ring.finish();
}

template <typename IO, int W, int NV, int R, bool ROWS>
int launch_stream(const QuantArgs& a, cudaStream_t stream) {
  constexpr int kGroups = kRingWarps / W;
  static PerDeviceOnce once;
  return launch_ring(quantize_stream_kernel<IO, W, NV, R, ROWS>, once,
                     (unsigned)ring_grid(a.rows, R, kGroups, a.panels, q8_sms()),
                     (size_t)a.panel * sizeof(IO) * R * kGroups, (size_t)a.panel * (ROWS && a.fold_cols ? 8 : 4), stream, a);
}

// Widest row that one group holds with codes by row: 16 warps, 32 elements (bf16) or 16 per thread.
template <typename IO>
constexpr int kWidest = sizeof(IO) == 2 ? 16384 : 8192;

template <typename IO, bool ROWS>
int run_stream(QuantArgs a, cudaStream_t stream) {
  a.panels = ROWS ? 1 : stream_panels(a.cols);
  a.panel = stream_panel(a.cols, a.panels);
  if constexpr (sizeof(IO) == 2) {
    // two rows of two octs up to 4096 columns (16384 x 2048: 36.3 us against 38.4 with one row of four),
    // one row of four beyond (4096 x 5120 both ways: 35.7 us against 41.9)
    if (ROWS && a.panel > 8192) return launch_stream<IO, 16, 4, 1, ROWS>(a, stream);
    if (a.panel > 4096) return launch_stream<IO, 8, 4, 1, ROWS>(a, stream);
  }
  return with_ring_warps(
      a.panel, [&](auto w) { return launch_stream<IO, decltype(w)::value, 2, kRingRows<IO>, ROWS>(a, stream); });
}

template <typename IO, int LANES>
int launch_panels(const QuantArgs& a, cudaStream_t stream) {
  // as many blocks as there are turns' worth of rows
  unsigned blocks = 1;
  while (blocks < kPanelCluster && a.rows > (int64_t)blocks * kPanelRows * (kPanelThreads / LANES)) blocks *= 2;
  return q8_code(launch_after(quantize_panel_kernel<IO, LANES>,
                              (unsigned)((a.cols + LANES * 8 - 1) / (LANES * 8)) * blocks, kPanelThreads, 0, stream, blocks,
                              a));
}
// 16 octs are 256 bytes of a bf16 row, and 1024 rows in one turn of a cluster of eight blocks; more rows are
// done sooner by 8 octs, which take twice the rows in a turn and have twice the clusters (1100 x 512: 3.8 us
// against 5.8, 4096 x 2048: 10.6 against 15.4; 1000 x 512: 4.3 against 4.2).  Beyond 2048 columns 16 octs fill
// the GPU with fewer, larger pieces (2048 x 4096: 10.1 us against 13.7).
template <typename IO>
int run_panels(const QuantArgs& a, cudaStream_t stream) {
  return a.cols <= 2048 && a.rows >= 1024 ? launch_panels<IO, 8>(a, stream) : launch_panels<IO, 16>(a, stream);
}

template <typename IO, int NV, int TPR>
int launch_rows(const QuantArgs& a, cudaStream_t stream) {
  constexpr int kRows = TPR <= 32 ? 256 / TPR : 1;
  return q8_code(launch_after(quantize_rows_kernel<IO, NV, TPR>, (unsigned)((a.rows + kRows - 1) / kRows),
                              TPR <= 32 ? 256 : TPR, 0, stream, 0, a));
}

template <typename IO>
int run_rows(const QuantArgs& a, bool octs, cudaStream_t stream) {
  const int c = a.cols;
  if (octs && c <= 16384) {
    if (c <= 64) return launch_rows<IO, 1, 8>(a, stream);
    if (c <= 128) return launch_rows<IO, 1, 16>(a, stream);
    if (c <= 256) return launch_rows<IO, 1, 32>(a, stream);
    if (c <= 512) return launch_rows<IO, 2, 32>(a, stream);
    if (c <= 1024) return launch_rows<IO, 4, 32>(a, stream);   // 16384 x 1024: 9.8 us, a block per row 17.7
    if (c <= 2048) return launch_rows<IO, 2, 128>(a, stream);
    if (c <= 4096) return launch_rows<IO, 2, 256>(a, stream);
    if (c <= 8192) return launch_rows<IO, 2, 512>(a, stream);
    return launch_rows<IO, 2, 1024>(a, stream);
  }
  auto go = [&](auto kernel, int per_block, int threads) {
    return q8_code(launch_after(kernel, (unsigned)((a.rows + per_block - 1) / per_block), (unsigned)threads, 0, stream, 0, a));
  };
  if (c + 7 <= 32768 && a.ld_qr % 8 == 0 && ((uintptr_t)a.q_rows & 7) == 0) {
    const int w = c + 7;                  // a row may need one more oct
    if (w <= 256) return go(quantize_rows_shifted_kernel<IO, 1, 32>, 8, 256);
    if (w <= 512) return go(quantize_rows_shifted_kernel<IO, 2, 32>, 8, 256);
    if (w <= 1024) return go(quantize_rows_shifted_kernel<IO, 1, 128>, 1, 128);
    if (w <= 2048) return go(quantize_rows_shifted_kernel<IO, 2, 128>, 1, 128);
    if (w <= 3072) return go(quantize_rows_shifted_kernel<IO, 3, 128>, 1, 128);
    if (w <= 4096) return go(quantize_rows_shifted_kernel<IO, 2, 256>, 1, 256);
    if (w <= 6144) return go(quantize_rows_shifted_kernel<IO, 3, 256>, 1, 256);
    if (w <= 8192) return go(quantize_rows_shifted_kernel<IO, 2, 512>, 1, 512);
    if (w <= 12288) return go(quantize_rows_shifted_kernel<IO, 3, 512>, 1, 512);
    if (w <= 16384) return go(quantize_rows_shifted_kernel<IO, 2, 1024>, 1, 1024);
    if (w <= 24576) return go(quantize_rows_shifted_kernel<IO, 3, 1024>, 1, 1024);
    return go(quantize_rows_shifted_kernel<IO, 4, 1024>, 1, 1024);
  }
  return c <= 1024 ? go(quantize_rows_single_kernel<IO, 128>, 1, 128) : go(quantize_rows_single_kernel<IO, 1024>, 1, 1024);
}

// Columns of any alignment.  (Octs aligned in memory, as the row kernels walk them, were slower here: the
// rows that start alike lie eight rows apart, 8192 x 4097 102 us against 77.)
template <typename IO>
int run_cols(const QuantArgs& a, cudaStream_t stream) {
  const int bx = (a.cols + kColThreads - 1) / kColThreads;
  // enough slabs for about eight blocks per SM, none shorter than 16 rows
  int64_t slabs = std::max<int64_t>(1, std::min<int64_t>((a.rows + 15) / 16, (8 * kRingBlocks + bx - 1) / bx));
  slabs = std::min<int64_t>(slabs, 65535);
  const int slab = (int)((a.rows + slabs - 1) / slabs);
  const dim3 grid((unsigned)bx, (unsigned)((a.rows + slab - 1) / slab));
  cudaError_t e = cudaMemsetAsync(a.top, 0, (size_t)a.cols * 4, stream);
  if (e == cudaSuccess) e = launch_in_turn(column_top_kernel<IO>, grid, kColThreads, stream, a, slab);
  if (e == cudaSuccess) e = launch_in_turn(quantize_cols_kernel<IO>, grid, kColThreads, stream, a, slab);
  return q8_code(e);
}

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" size_t prm_quantize_q8_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1) return 0;
  // the columns' maxima, and those of every block's rows
  return ((size_t)std::min<int64_t>(rows, kRingBlocks) + 1) * ((size_t)cols + 256) * 4;
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
  if (((uintptr_t)scale_rows | (uintptr_t)scale_cols | (uintptr_t)fold_rows | (uintptr_t)fold_cols) % 4 != 0 ||
      (q_cols && !aligned16(scratch)))
    return PRM_ERR_ALIGN;
  if (rows == 0) {                        // columns without an element: scale 0
    return q_cols ? q8_code(cudaMemsetAsync(scale_cols, 0, (size_t)cols * 4, stream)) : PRM_OK;
  }
  if (!x) return PRM_ERR_ARG;
  if ((uintptr_t)x % (io_fp32 ? 4 : 2) != 0) return PRM_ERR_ALIGN;
  if (q_cols && (!scratch || scratch_bytes < prm_quantize_q8_scratch_bytes(rows, cols))) return PRM_ERR_WORKSPACE;
  QuantArgs a = {x, fold_rows, fold_cols, (uint8_t*)q_rows, (uint8_t*)q_cols, scale_rows, scale_cols,
                 (uint32_t*)scratch, (float*)scratch + (cols + 7) / 8 * 8, rows, ld_x, ld_q_rows, ld_q_cols, (int)cols, format};
  const bool octs_x = cols % 8 == 0 && ld_x % 8 == 0 && aligned16(x);
  const bool octs_r = octs_x && ld_q_rows % 8 == 0 && ((uintptr_t)q_rows & 7) == 0;
  const bool octs_c = octs_x && ld_q_cols % 8 == 0 && ((uintptr_t)q_cols & 7) == 0;
  // Codes by column of an aligned matrix: one launch, with the codes by row in the same pass where a
  // row fits a group's registers.
  // Up to these sizes by panels (1500 x 2048 both ways with folds: 10.5 us, streamed 19.2; 4096 x 4096 columns:
  // 17.7 against 22.5), beyond them streamed (8192 x 8192: 58.8 against 67.5; 32768 x 512: 28.5 against 45.1).
  const bool panels = q_cols && octs_c && rows <= (cols < 256 ? 2048 : 8192) && rows * cols <= (int64_t)1 << 24;
  int code = PRM_OK;
  if (panels) {
    code = io_fp32 ? run_panels<float>(a, stream) : run_panels<__nv_bfloat16>(a, stream);
    q_cols = nullptr;
  } else if (q_cols && octs_c && stream_takes(cols, q8_sms())) {
    const bool joint = q_rows && octs_r && cols <= (io_fp32 ? kWidest<float> : kWidest<__nv_bfloat16>);
    if (joint) code = io_fp32 ? run_stream<float, true>(a, stream) : run_stream<__nv_bfloat16, true>(a, stream);
    else code = io_fp32 ? run_stream<float, false>(a, stream) : run_stream<__nv_bfloat16, false>(a, stream);
    if (joint) q_rows = nullptr;
    q_cols = nullptr;
  }
  if (code == PRM_OK && q_rows)
    code = io_fp32 ? run_rows<float>(a, octs_r, stream) : run_rows<__nv_bfloat16>(a, octs_r, stream);
  if (code == PRM_OK && q_cols) code = io_fp32 ? run_cols<float>(a, stream) : run_cols<__nv_bfloat16>(a, stream);
  return code;
}
