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

// What a set of values with the largest magnitude `top` is multiplied by, and the scale that undoes
// it.  The factor is limit * (1 / top), each step rounded, which is how array libraries evaluate a
// number over an array: codes then agree bit for bit with `(t * (limit / top)).round()` written
// there.  `top_bits` is the maximum of the magnitudes' bit patterns as unsigned integers, which orders
// NaN above infinity above every number: a set that holds either gets the scale NaN and zero codes,
// so it marks its own row (column) of whatever is computed from it and no other.
struct Q8Scale {
  float mul, scale;
  bool finite;
};
__device__ __forceinline__ Q8Scale q8_scale(uint32_t top_bits, float limit) {
  Q8Scale s;
  const float top = __uint_as_float(top_bits);
  s.finite = top_bits < 0x7f800000u;
  const bool live = s.finite && top >= kQ8Tiny;
  s.mul = live ? __fmul_rn(limit, __frcp_rn(top)) : 0.f;
  s.scale = live ? __fdiv_rn(top, limit) : (s.finite ? 0.f : __uint_as_float(0x7fc00000u));
  return s;
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Four values, already multiplied, to four codes (first value in the lowest byte).
__device__ __forceinline__ uint32_t q8_pack4(float a, float b, float c, float d, int format) {
  if (format == PRM_Q8_INT8) {
    // |v| <= 127: adding 1.5 * 2^23 leaves the value rounded to nearest-even in the low bits.
    const float m = 12582912.f;
    const uint32_t x = __float_as_uint(__fadd_rn(a, m)), y = __float_as_uint(__fadd_rn(b, m));
    const uint32_t z = __float_as_uint(__fadd_rn(c, m)), w = __float_as_uint(__fadd_rn(d, m));
    return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
  }
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
__device__ __forceinline__ uint8_t q8_pack1(float a, int format) {
  return (uint8_t)(q8_pack4(a, 0.f, 0.f, 0.f, format) & 0xffu);
}

// VEC consecutive elements as fp32 (VEC = 8: 16-byte aligned; VEC = 1: anywhere).
template <int VEC, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&out)[VEC]) {
  if constexpr (VEC == 8) {
    load8(p, out);
  } else {
    out[0] = to_f32(*p);
  }
}
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&in)[VEC]) {
  if constexpr (VEC == 8) {
    store8(p, in);
  } else {
    from_f32(p, in[0]);
  }
}
template <int VEC>
__device__ __forceinline__ void load_weight(const void* w, int fp32, int64_t i, float (&out)[VEC]) {
  if (fp32) {
    load_vec<VEC>(reinterpret_cast<const float*>(w) + i, out);
  } else {
    load_vec<VEC>(reinterpret_cast<const __nv_bfloat16*>(w) + i, out);
  }
}
template <int VEC>
__device__ __forceinline__ void store_codes(uint8_t* p, const float (&v)[VEC], int format) {
  if constexpr (VEC == 8) {
    uint2 c;
    c.x = q8_pack4(v[0], v[1], v[2], v[3], format);
    c.y = q8_pack4(v[4], v[5], v[6], v[7], format);
    *reinterpret_cast<uint2*>(p) = c;
  } else {
    *p = q8_pack1(v[0], format);
  }
}
// The value as it is kept in the stream's type.
__device__ __forceinline__ float as_stored(float v, const float*) { return v; }
__device__ __forceinline__ float as_stored(float v, const __nv_bfloat16*) {
  return __bfloat162float(__float2bfloat16_rn(v));
}

// Sum and (unsigned) maximum over the first `THREADS` threads of a block of exactly that size;
// every thread gets both.  `red` holds 2 * 32 words and may be used again after the next call's
// first barrier (calls alternate between two arrays).
template <int THREADS>
__device__ __forceinline__ void block_sum_max(float& sum, uint32_t& top, uint32_t* red) {
  sum = warp_sum(sum);
  top = __reduce_max_sync(0xffffffffu, top);
  if constexpr (THREADS > 32) {
    constexpr int kWarps = THREADS / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
      red[warp] = __float_as_uint(sum);
      red[32 + warp] = top;
    }
    __syncthreads();
    sum = lane < kWarps ? __uint_as_float(red[lane]) : 0.f;
    top = lane < kWarps ? red[32 + lane] : 0u;
    sum = warp_sum(sum);
    top = __reduce_max_sync(0xffffffffu, top);
  }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace prm
