// 8-bit operators around a linear layer: what the norm, the quantiser and the product share.
//
// A quantised matrix is a matrix of 8-bit codes with one fp32 scale per row or per column, value =
// code * scale.  Codes are int8 in [-127, 127] or e4m3 in [-448, 448]; the largest magnitude that
// shares a scale maps to the limit, so a code is the value times limit / largest, rounded to
// nearest-even in the format.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "launch.cuh"

namespace prm {

constexpr float kLimitInt8 = 127.f;
constexpr float kLimitE4m3 = 448.f;
// Below this a largest magnitude counts as zero (all codes and the scale are 0): limit / largest
// would leave the fp32 range from 2^-119 on.
constexpr float kQ8Tiny = 0x1p-100f;

__host__ __device__ inline bool q8_format_ok(int format) { return format == PRM_Q8_INT8 || format == PRM_Q8_E4M3; }
__host__ __device__ inline float q8_limit(int format) { return format == PRM_Q8_INT8 ? kLimitInt8 : kLimitE4m3; }

// A set of values with the largest magnitude `top` is multiplied by q8_mul and marked with q8_scale,
// which undoes it.  The factor is limit * (1 / top) and a code the rounded product, each step rounded to
// fp32, which is how array libraries evaluate `round(t * (limit / top))` with a number over an array.
// A set that holds an infinity or a NaN (which maxima here keep) gets the scale NaN and zero codes: it
// marks its own row (column) of whatever is computed from it and no other.
__device__ __forceinline__ bool q8_finite(float top) { return top < __uint_as_float(0x7f800000u); }
__device__ __forceinline__ float q8_mul(float top, float limit) {
  return top >= kQ8Tiny && q8_finite(top) ? __fmul_rn(limit, __frcp_rn(top)) : 0.f;
}
__device__ __forceinline__ float q8_scale(float top, float limit) {
  return !q8_finite(top) ? __uint_as_float(0x7fc00000u) : top >= kQ8Tiny ? __fdiv_rn(top, limit) : 0.f;
}

// ------------------------------------------------------------- eight elements at a time
// The row operators read 2 to 6 bytes per element, so what bounds them next to memory is the number
// of instructions per element: everything below works on pairs (fp32x2 products, sums and fused
// products round like their scalar forms; bf16x2 conversions; a three-way maximum).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
// Largest of m and the two magnitudes; a NaN among them stays.
__device__ __forceinline__ float max_abs(float m, float2 v) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(m), "f"(fabsf(v.x)), "f"(fabsf(v.y)));
  return d;
}
__device__ __forceinline__ float2 pair_of(uint32_t bf16x2) {
  return make_float2(__uint_as_float(bf16x2 << 16), __uint_as_float(bf16x2 & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pair_to_bf16(float2 v) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  return reinterpret_cast<const uint32_t&>(h);
}

// Eight elements as stored (16-byte aligned), converted on use, so that a kernel that takes several
// has all its loads under way before it waits for the first.
template <typename T> struct Oct;
template <> struct Oct<__nv_bfloat16> {
  uint4 r;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load_stream(const __nv_bfloat16* p) { r = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = r; }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
    v[0] = pair_of(r.x);
    v[1] = pair_of(r.y);
    v[2] = pair_of(r.z);
    v[3] = pair_of(r.w);
  }
  __device__ __forceinline__ void set(const float2 (&v)[4]) {
    r = make_uint4(pair_to_bf16(v[0]), pair_to_bf16(v[1]), pair_to_bf16(v[2]), pair_to_bf16(v[3]));
  }
  __device__ __forceinline__ void zero() { r = make_uint4(0, 0, 0, 0); }
};
template <> struct Oct<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void load_stream(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p + 4));
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<float4*>(p) = a;
    *reinterpret_cast<float4*>(p + 4) = b;
  }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
    v[0] = make_float2(a.x, a.y);
    v[1] = make_float2(a.z, a.w);
    v[2] = make_float2(b.x, b.y);
    v[3] = make_float2(b.z, b.w);
  }
  __device__ __forceinline__ void set(const float2 (&v)[4]) {
    a = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    b = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
};

// The int8 codes of t * mul in the low bytes: |t * mul| <= 127, and adding 1.5 * 2^23 leaves it rounded to
// nearest-even there.  The product has to be rounded before: in one fused step 1 in 2,700 bf16 values, next
// to a tie, gets another code than by the rule above.  A product and a sum of pairs come out of the
// assembler as one fused step, explicit rounding or not, so the product is itself a fused step, with a -0
// that the assembler does not take for a known number: `nz` comes with the kernel's arguments (from
// constant memory one token of the norm takes 1.9 us instead of 1.6).
__device__ __forceinline__ float2 int8_bits(float2 t, float2 mul, float nz) {
  return add2(fma2(t, mul, make_float2(nz, nz)), make_float2(12582912.f, 12582912.f));
}
// Four codes of t * mul (first value in the lowest byte).
template <int FORMAT>
__device__ __forceinline__ uint32_t codes4(float2 a, float2 b, float2 mul, float nz) {
  if constexpr (FORMAT == PRM_Q8_INT8) {
    a = int8_bits(a, mul, nz);
    b = int8_bits(b, mul, nz);
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                       __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
  } else {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(mul2(a, mul), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(mul2(b, mul), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  }
}
__device__ __forceinline__ uint8_t code1(float v, float mul, int format) {
  if (format == PRM_Q8_INT8) return (uint8_t)__float_as_uint(__fadd_rn(__fmul_rn(v, mul), 12582912.f));
  return (uint8_t)__nv_cvt_float_to_fp8(__fmul_rn(v, mul), __NV_SATFINITE, __NV_E4M3);
}
// The codes of NV octs of a thread, `stride` elements apart, below `cols`; zeros where the row has no
// number for a scale.
template <int NV, int FORMAT>
__device__ __forceinline__ void store_octs_as(uint8_t* q, const float2 (&t)[NV][4], int c0, int stride, int cols,
                                              float top, float nz) {
  const float f = q8_mul(top, q8_limit(FORMAT));
  const float2 mul = make_float2(f, f);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * stride;
    if (c < cols)
      *reinterpret_cast<uint2*>(q + c) =
          make_uint2(codes4<FORMAT>(t[v][0], t[v][1], mul, nz), codes4<FORMAT>(t[v][2], t[v][3], mul, nz));
  }
}
template <int NV>
__device__ __forceinline__ void store_octs(uint8_t* q, const float2 (&t)[NV][4], int c0, int stride, int cols,
                                           float top, int format, float nz) {
  if (!q8_finite(top)) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (c0 + v * stride < cols) *reinterpret_cast<uint2*>(q + c0 + v * stride) = make_uint2(0u, 0u);
  } else if (format == PRM_Q8_INT8) {
    store_octs_as<NV, PRM_Q8_INT8>(q, t, c0, stride, cols, top, nz);
  } else {
    store_octs_as<NV, PRM_Q8_E4M3>(q, t, c0, stride, cols, top, nz);
  }
}

// ---------------------------------------------- rows that do not start on an oct's boundary
// A row is walked through in octs that are aligned in memory: oct o holds elements 8 o - shift .. 8 o -
// shift + 7, `shift` = what the row's start lies behind a boundary, alike for all matrices that are
// walked together.  Octs that reach over either end of the row go element by element.
template <typename T>
__host__ __device__ __forceinline__ int oct_shift(const T* row) {
  return (int)(((uintptr_t)row / sizeof(T)) & 7);
}
// One row of a matrix as the octs see it: the elements before and behind it that belong to the same
// matrix may be fetched along (an oct at the end of a row is one load like all others, and nothing
// waits for it before the other loads are under way), nothing beyond the matrix is.
template <typename T>
struct OctRow {
  const T* p;
  int before, after;                       // elements of the matrix before the row's start (8 are enough), and from it on
  __device__ __forceinline__ OctRow(const void* base, int64_t row, int64_t rows, int64_t ld, int cols)
      : p(reinterpret_cast<const T*>(base) + row * ld),
        before((int)min((int64_t)8, row * ld)),
        after((int)min((int64_t)cols + 8, (rows - 1 - row) * ld + cols)) {}
  __device__ __forceinline__ void load(int first, int cols, Oct<T>& o) const {
    if (first >= cols) {
      o.zero();
    } else if (first + before >= 0 && first + 8 <= after) {
      o.load_stream(p + first);
    } else {
      float2 v[4];
      float e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = first + k >= 0 && first + k < cols ? to_f32(p[first + k]) : 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = make_float2(e[2 * k], e[2 * k + 1]);
      o.set(v);
    }
  }
};
// The oct's elements that lie in the row, zeros for the others.
template <typename T>
__device__ __forceinline__ void get_part(const Oct<T>& o, int first, int cols, float2 (&v)[4]) {
  o.get(v);
  if (first < 0 || first + 8 > cols) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (first + 2 * k < 0 || first + 2 * k >= cols) v[k].x = 0.f;
      if (first + 2 * k + 1 < 0 || first + 2 * k + 1 >= cols) v[k].y = 0.f;
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_part(T* row, int first, int cols, const float2 (&v)[4]) {
  if (first >= 0 && first + 8 <= cols) {
    Oct<T> o;
    o.set(v);
    o.store(row + first);
  } else if (first < cols) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (first + k >= 0 && first + k < cols) from_f32(row + first + k, k & 1 ? v[k / 2].y : v[k / 2].x);
  }
}
// Eight factors from `first` on of a vector of any alignment (0 outside it).  Inside it the loads have no
// conditions, so that they are under way together.
template <typename T>
__device__ __forceinline__ void load_factors(const T* f, int first, int cols, float2 (&v)[4]) {
  if (first >= 0 && first + 8 <= cols) {
    const T* p = f + first;
    if (((uintptr_t)p & 15) == 0) {
      Oct<T> o;
      o.load(p);
      o.get(v);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = make_float2(to_f32(p[2 * k]), to_f32(p[2 * k + 1]));
    }
  } else if (first >= cols) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float2(0.f, 0.f);
  } else {
    float e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) e[k] = first + k >= 0 && first + k < cols ? to_f32(f[first + k]) : 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float2(e[2 * k], e[2 * k + 1]);
  }
}
__device__ __forceinline__ void load_factors(const void* f, int fp32, int first, int cols, float2 (&v)[4]) {
  if (fp32) load_factors(reinterpret_cast<const float*>(f), first, cols, v);
  else load_factors(reinterpret_cast<const __nv_bfloat16*>(f), first, cols, v);
}
// The codes of a row's octs (NV per thread of TPR) to a row of codes whose start is 8-byte aligned.  Word
// k of it is made of the end of oct k and the beginning of oct k + 1, which another thread holds: the
// octs meet in `stage`, NV * TPR + 1 words of shared memory.
template <int NV, int TPR>
__device__ __forceinline__ void store_octs_shifted(uint64_t* stage, uint8_t* q, const float2 (&t)[NV][4], int o0,
                                                   int shift, int cols, float top, int format, float nz) {
  const bool finite = q8_finite(top);
  const float f = q8_mul(top, q8_limit(format));
  const float2 mul = make_float2(f, f);
  uint64_t c[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    uint2 w = make_uint2(0u, 0u);
    if (finite)
      w = format == PRM_Q8_INT8 ? make_uint2(codes4<PRM_Q8_INT8>(t[v][0], t[v][1], mul, nz), codes4<PRM_Q8_INT8>(t[v][2], t[v][3], mul, nz))
                                : make_uint2(codes4<PRM_Q8_E4M3>(t[v][0], t[v][1], mul, nz), codes4<PRM_Q8_E4M3>(t[v][2], t[v][3], mul, nz));
    c[v] = (uint64_t)w.x | ((uint64_t)w.y << 32);
  }
  if (shift) {                             // alike for all threads of the row
#pragma unroll
    for (int v = 0; v < NV; ++v) stage[o0 + v * TPR] = c[v];
    if constexpr (TPR == 32) __syncwarp();
    else __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; ++v) c[v] = (c[v] >> (8 * shift)) | (stage[o0 + v * TPR + 1] << (64 - 8 * shift));
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int word = (o0 + v * TPR) * 8;
    if (word + 8 <= cols) {
      *reinterpret_cast<uint64_t*>(q + word) = c[v];
    } else {
      for (int k = 0; word + k < cols; ++k) q[word + k] = (uint8_t)(c[v] >> (8 * k));
    }
  }
}
// Whether rows of the two matrices start alike: then their octs are aligned together.
template <typename T>
inline bool octs_alike(const void* p, int64_t ld_p, const void* q, int64_t ld_q) {
  return oct_shift((const T*)p) == oct_shift((const T*)q) && ((ld_p - ld_q) & 7) == 0 &&
         ((uintptr_t)p % sizeof(T)) == 0 && ((uintptr_t)q % sizeof(T)) == 0;
}

__device__ __forceinline__ float load1(const void* p, int fp32, int64_t i) {
  return fp32 ? reinterpret_cast<const float*>(p)[i] : to_f32(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
}
// The value as it is kept in the stream's type.
__device__ __forceinline__ float as_stored(float v, const float*) { return v; }
__device__ __forceinline__ float as_stored(float v, const __nv_bfloat16*) {
  return __bfloat162float(__float2bfloat16_rn(v));
}

// Sum over groups of N neighbouring lanes of a warp, for each of them.
template <int N>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Largest value over the same; a NaN in any lane stays (`top` is no negative number).
template <int N = 32>
__device__ __forceinline__ float group_top(float top) {
  uint32_t v = __float_as_uint(top);
  if constexpr (N == 32) {
    v = __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  }
  return __uint_as_float(v);
}
// Sum and largest magnitude over a block of THREADS threads (up to 32: groups of lanes); every thread
// gets both.  `red`: 64 words, used once between two barriers.
template <int THREADS>
__device__ __forceinline__ void block_sum_top(float& sum, float& top, float* red) {
  sum = group_sum<(THREADS < 32 ? THREADS : 32)>(sum);
  top = group_top<(THREADS < 32 ? THREADS : 32)>(top);
  if constexpr (THREADS > 32) {
    constexpr int kWarps = THREADS / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
      red[warp] = sum;
      red[32 + warp] = top;
    }
    __syncthreads();
    sum = lane < kWarps ? red[lane] : 0.f;
    top = lane < kWarps ? red[32 + lane] : 0.f;
    sum = warp_sum(sum);
    top = group_top(top);
  }
}

// Sums of two numbers over a block of THREADS threads.  `red`: 64 words; calls in turn use two sets.
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

// Launches that overlap the end of the kernel before them (programmatic dependent launch): every
// kernel that is launched so calls grid_wait() before it touches global memory, which holds it until all kernels
// before it in the stream have finished and their writes are visible, and grid_trigger() once it
// holds all resources that it will ever ask for, which lets the next kernel start setting up.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
inline cudaError_t launch_after(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, cudaStream_t stream,
                                unsigned cluster, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(block, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// The same without the overlap and without clusters.
template <typename... P, typename... A>
inline cudaError_t launch_in_turn(void (*kernel)(P...), dim3 grid, unsigned block, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block, 1, 1);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// What a call returns for its own CUDA calls: not what an earlier one has left as the thread's last error,
// and leaving none behind for those who ask for it.
inline int q8_code(cudaError_t e) {
  if (e == cudaSuccess) return PRM_OK;
  cudaGetLastError();
  return PRM_ERR_CUDA;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace prm
