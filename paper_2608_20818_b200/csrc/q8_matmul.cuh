// What the two kernels of the 8-bit product share: the problem, its tensor maps, the choice.
#pragma once

#include <cmath>

#include "q8.cuh"
#include "tcgen05.cuh"

namespace prm {

constexpr int kBlockK = 128;           // one 128-byte swizzled row of k
// 32-bit sums of products of int8 hold for this many k-blocks (2^14 * 128 * 1023 < 2^31); longer
// sums are split over a cluster, whose parts are added in 64 bits.
constexpr int kMaxBlocksInt8 = 1023;

// What both kernels read besides their tensor maps.
struct MatmulArgs {
  const float* scale_a;   // [m] or null
  const float* scale_b;   // [n] or null
  void* out;
  int* status;
  int64_t ld_out;
  int m, n;
  int kblocks;            // ceil(k / 128)
  int out_fp32;
};

// Up to ROWS rows of one output column per lane; `sa` is the scale of row `lane` of these.  All rows
// are scaled before the first store and full sets are stored without a test per row: with one the
// rows follow one another at the latency of a shuffle, two products and a store each (12,400 cycles
// for a 256 x 256 tile of a CTA pair).
template <bool INT8, int ROWS, typename OUT>
__device__ __forceinline__ void store_column(OUT* out, int64_t ld, const uint32_t (&r)[ROWS], float sa, float sb,
                                             int rows, bool live) {
  float v[ROWS];
#pragma unroll
  for (int j = 0; j < ROWS; ++j)
    v[j] = (INT8 ? (float)(int)r[j] : __uint_as_float(r[j])) * __shfl_sync(0xffffffffu, sa, j) * sb;
  if (!live) return;
  if (rows >= ROWS) {
#pragma unroll
    for (int j = 0; j < ROWS; ++j) from_f32(out + j * ld, v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
      if (j < rows) from_f32(out + j * ld, v[j]);
  }
}

// The status word that prm_q8_status reads, on the current device (null if it has none).
int* q8_status_word();

struct MatmulProblem {
  MatmulArgs c;
  const void *a, *b;
  int64_t ld_a, ld_b, a_rows, a_cols, b_rows, b_cols;   // as stored
  bool a_t, b_t;          // stored k x m, n x k
  bool int8;
  cudaStream_t stream;
};

// Pairs of CTAs on 256 x 256 tiles, for products that fill the GPU with them.
// Estimated SM cycles, without what every launch costs.
double matmul_q8_pairs_cycles(const MatmulProblem& p);
int matmul_q8_pairs(const MatmulProblem& p);

typedef CUresult (*Q8EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline Q8EncodeFn q8_encode_fn() {
  static Q8EncodeFn fn = []() -> Q8EncodeFn {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult res;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &res) != cudaSuccess ||
        res != cudaDriverEntryPointSuccess)
      return nullptr;
    return (Q8EncodeFn)p;
  }();
  return fn;
}

// Map over rows x cols bytes (row-major, ld bytes apart), boxes of box_rows x 128 bytes; what lies
// outside reads as zero.
inline bool q8_make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  Q8EncodeFn encode = q8_encode_fn();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Cycles that HBM needs for the operands at 6.4 TB/s and 1.9 GHz.
inline double matmul_q8_memory_cycles(const MatmulProblem& p) {
  return ((double)p.a_rows * p.a_cols + (double)p.b_rows * p.b_cols) / 3400.0;
}

// Clusters of `size` CTAs that can be resident at once (0: an error).
template <typename K>
inline int q8_resident_clusters(K kernel, unsigned threads, size_t smem, unsigned size) {
  int dev = 0, sms = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)sms / size * size, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess ? n : 0;
}

}  // namespace prm
