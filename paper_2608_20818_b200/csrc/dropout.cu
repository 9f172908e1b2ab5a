// out = x dropped out (+ residual); applied to a gradient with the same numbers it is its own gradient.
//
// Bound by HBM (2 or 3 elements' bytes each) and by the generator's integer products and exclusive ors, which do not
// overlap well with one another: 8192 x 8192 in bf16 61 us, with residual 67 us (6.0 TB/s); in fp32 89 and 118 us (6.0, 6.8).
// A block takes 256 / TPR rows (TPR threads to a row) by 4 TPR
// octs; a thread's four octs are under way together.
#include "dropout.cuh"

namespace prm {
namespace {

struct DropoutArgs {
  const void* x;
  const void* residual;    // may be null
  void* out;
  int64_t rows, ld_x, ld_r, ld_out;
  int cols;
  int chunks;              // of columns
  Drop drop;
};

constexpr int kOcts = 4;                   // per thread

// SHIFT: octs aligned in memory of rows that start anywhere (alike in all matrices); an oct may then need the words of
// three quads (8192 x 8191: 111 us).
template <typename IO, int TPR, bool SHIFT>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs a) {
  grid_wait();
  grid_trigger();
  const int chunk = blockIdx.x % (unsigned)a.chunks;
  const int64_t row = (int64_t)(blockIdx.x / (unsigned)a.chunks) * (256 / TPR) + threadIdx.x / TPR;
  if (row >= a.rows) return;
  const uint64_t number = drop_number(a.drop);
  const OctRow<IO> x(a.x, row, a.rows, a.ld_x, a.cols);
  const OctRow<IO> r(a.residual ? a.residual : a.x, row, a.rows, a.residual ? a.ld_r : a.ld_x, a.cols);
  IO* out = reinterpret_cast<IO*>(a.out) + row * a.ld_out;
  const int shift = SHIFT ? oct_shift(x.p) : 0;
  const int c0 = (chunk * kOcts * TPR + (int)(threadIdx.x % TPR)) * 8 - shift;
  Oct<IO> xv[kOcts], rv[kOcts];
#pragma unroll
  for (int k = 0; k < kOcts; ++k) {
    const int c = c0 + k * TPR * 8;
    if (c < a.cols) {
      if constexpr (SHIFT) {
        x.load(c, a.cols, xv[k]);
        if (a.residual) r.load(c, a.cols, rv[k]);
      } else {
        xv[k].load_stream(x.p + c);
        if (a.residual) rv[k].load_stream(r.p + c);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kOcts; ++k) {
    const int c = c0 + k * TPR * 8;
    if (c < a.cols) {
      float2 v[4], b[4];
      xv[k].get(v);
      drop_oct<!SHIFT>(a.drop, number, (uint32_t)row, c, v);
      if (a.residual) {
        rv[k].get(b);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = add2(v[e], b[e]);
      }
      if constexpr (SHIFT) {
        store_part(out, c, a.cols, v);
      } else {
        xv[k].set(v);
        xv[k].store(out + c);
      }
    }
  }
}

// Matrices whose rows start unlike one another: four elements per thread, one by one.
template <typename IO>
__global__ void __launch_bounds__(256) dropout_single_kernel(const DropoutArgs a) {
  grid_wait();
  grid_trigger();
  const int64_t row = blockIdx.x / (unsigned)a.chunks;
  const int c0 = (int)(blockIdx.x % (unsigned)a.chunks) * 1024 + (int)threadIdx.x * 4;
  if (c0 >= a.cols) return;
  const IO* x = reinterpret_cast<const IO*>(a.x) + row * a.ld_x;
  const IO* r = a.residual ? reinterpret_cast<const IO*>(a.residual) + row * a.ld_r : nullptr;
  IO* out = reinterpret_cast<IO*>(a.out) + row * a.ld_out;
  const uint4 w = drop_words(a.drop, drop_number(a.drop), (uint32_t)row, (uint32_t)c0 >> 2);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (c0 + k < a.cols) {
      const float v = dropped(a.drop, word[k], to_f32(x[c0 + k]));
      from_f32(out + c0 + k, r ? v + to_f32(r[c0 + k]) : v);
    }
  }
}

template <typename IO, int TPR, bool SHIFT>
int launch_dropout(DropoutArgs a, cudaStream_t stream) {
  const int octs = (a.cols + (SHIFT ? 7 : 0) + 7) / 8;
  a.chunks = (octs + kOcts * TPR - 1) / (kOcts * TPR);
  const int64_t blocks = (a.rows + 256 / TPR - 1) / (256 / TPR) * a.chunks;
  if (blocks > 0x7fffffffLL) return PRM_ERR_SHAPE;
  return q8_code(launch_after(dropout_kernel<IO, TPR, SHIFT>, (unsigned)blocks, 256, 0, stream, 0, a));
}
template <typename IO, bool SHIFT>
int run_dropout(const DropoutArgs& a, cudaStream_t stream) {
  if (a.cols <= 256) return launch_dropout<IO, 8, SHIFT>(a, stream);
  if (a.cols <= 1024) return launch_dropout<IO, 32, SHIFT>(a, stream);
  return launch_dropout<IO, 256, SHIFT>(a, stream);
}
template <typename IO>
int run_any(DropoutArgs a, cudaStream_t stream) {
  const bool octs = a.cols % 8 == 0 && a.ld_x % 8 == 0 && a.ld_out % 8 == 0 && aligned16(a.x) && aligned16(a.out) &&
                    (!a.residual || (a.ld_r % 8 == 0 && aligned16(a.residual)));
  if (octs) return run_dropout<IO, false>(a, stream);
  if (octs_alike<IO>(a.x, a.ld_x, a.out, a.ld_out) && (!a.residual || octs_alike<IO>(a.x, a.ld_x, a.residual, a.ld_r)))
    return run_dropout<IO, true>(a, stream);
  a.chunks = (a.cols + 1023) / 1024;
  if (a.rows * a.chunks > 0x7fffffffLL) return PRM_ERR_SHAPE;
  return q8_code(launch_after(dropout_single_kernel<IO>, (unsigned)(a.rows * a.chunks), 256, 0, stream, 0, a));
}

bool ld_ok(int64_t ld) { return ld >= 0 && ld <= ((int64_t)1 << 40); }

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" int prm_dropout(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int64_t rows,
                           int64_t cols, int io_fp32, double p, uint64_t seed, uint64_t offset,
                           const uint64_t* counter, void* out, int64_t ld_out, void* cuda_stream) {
  if (!drop_ok(p) || rows < 0) return PRM_ERR_ARG;
  if (cols < 0 || cols > 0x7fffffffLL - 8192 || rows > 0x7fffffffLL) return PRM_ERR_SHAPE;
  if (!ld_ok(ld_x) || (residual && !ld_ok(ld_residual)) || ld_out < cols || !ld_ok(ld_out)) return PRM_ERR_SHAPE;
  if (rows == 0 || cols == 0) return PRM_OK;
  if (!x || !out) return PRM_ERR_ARG;
  if (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)out) % (io_fp32 ? 4 : 2) != 0 || (uintptr_t)counter % 8 != 0)
    return PRM_ERR_ALIGN;
  DropoutArgs a = {x, residual, out, rows, ld_x, ld_residual, ld_out, (int)cols, 1, make_drop(p, seed, offset, counter)};
  return io_fp32 ? run_any<float>(a, (cudaStream_t)cuda_stream) : run_any<__nv_bfloat16>(a, (cudaStream_t)cuda_stream);
}
