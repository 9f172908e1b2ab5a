// Layer norm with the residual's addition and dropout: what its two directions share.
#pragma once

#include "dropout.cuh"
#include "train_plan.h"

namespace prm {

// SMs of the current device, 148 at most (0: an error).
int q8_sms();

// Scale and shift of a row: one row of them for all rows, or one for each group of `rows_per_group`.
struct Affine {
  const void* weight;      // may be null (1)
  const void* bias;        // may be null (0)
  int64_t ld_w, ld_b;
  int fp32;
  int add_one;             // the weight is 1 + what is stored
};

__device__ __forceinline__ void affine_weight(const Affine& a, int64_t group, int first, int cols, float2 (&w)[4]) {
  if (!a.weight) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = make_float2(1.f, 1.f);
    return;
  }
  const char* p = reinterpret_cast<const char*>(a.weight) + group * a.ld_w * (a.fp32 ? 4 : 2);
  load_factors(p, a.fp32, first, cols, w);
  if (a.add_one) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = add2(w[e], make_float2(1.f, 1.f));
  }
}
// Eight factors as stored, in either type.
struct RawFactors {
  uint4 lo, hi;
  __device__ __forceinline__ void load(const void* p, int fp32, int64_t at) {
    const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + at * (fp32 ? 4 : 2));
    lo = q[0];
    if (fp32) hi = q[1];
  }
  __device__ __forceinline__ void get(int fp32, float2 (&v)[4]) const {
    if (fp32) {
      v[0] = make_float2(__uint_as_float(lo.x), __uint_as_float(lo.y));
      v[1] = make_float2(__uint_as_float(lo.z), __uint_as_float(lo.w));
      v[2] = make_float2(__uint_as_float(hi.x), __uint_as_float(hi.y));
      v[3] = make_float2(__uint_as_float(hi.z), __uint_as_float(hi.w));
    } else {
      v[0] = pair_of(lo.x);
      v[1] = pair_of(lo.y);
      v[2] = pair_of(lo.z);
      v[3] = pair_of(lo.w);
    }
  }
};
__device__ __forceinline__ void affine_bias(const Affine& a, int64_t group, int first, int cols, float2 (&b)[4]) {
  if (!a.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = make_float2(0.f, 0.f);
    return;
  }
  const char* p = reinterpret_cast<const char*>(a.bias) + group * a.ld_b * (a.fp32 ? 4 : 2);
  load_factors(p, a.fp32, first, cols, b);
}
__device__ __forceinline__ float affine_weight1(const Affine& a, int64_t group, int c) {
  if (!a.weight) return 1.f;
  const float w = load1(a.weight, a.fp32, group * a.ld_w + c);
  return a.add_one ? 1.f + w : w;
}
__device__ __forceinline__ float affine_bias1(const Affine& a, int64_t group, int c) {
  return a.bias ? load1(a.bias, a.fp32, group * a.ld_b + c) : 0.f;
}

// Zeros for the oct's elements outside the row.
__device__ __forceinline__ void clear_outside(int first, int cols, float2 (&v)[4]) {
  if (first < 0 || first + 8 > cols) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (first + 2 * k < 0 || first + 2 * k >= cols) v[k].x = 0.f;
      if (first + 2 * k + 1 < 0 || first + 2 * k + 1 >= cols) v[k].y = 0.f;
    }
  }
}

inline bool layernorm_ld_ok(int64_t ld) { return ld >= 0 && ld <= ((int64_t)1 << 40); }

// Sums over a group of TPR of the block's threads.  Groups of several warps meet in `red` (a word per warp and
// number) at the group's own barrier; whoever calls this twice in turn with two buffers needs no other.
template <int TPR, int BLOCK>
__device__ __forceinline__ void group_barrier() {
  if constexpr (TPR == BLOCK) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.x / TPR + 1), "n"(TPR) : "memory");
}
// N (a power of two) sums at once over a warp: while there are several, a lane hands half of them to its partner and
// takes the partner's share of the others, so that N numbers cost N - 1 + log2(32 / N) shuffles, not 5 N.  The sum of
// number k is then in the lanes whose highest bits are k.
template <int N, int WIDTH>
__device__ __forceinline__ void lane_sums(float (&v)[N]) {
  if constexpr (N == 1 || WIDTH < 32) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = group_sum<WIDTH>(v[k]);
  } else {
    constexpr int kHalf = N / 2;
    const bool upper = threadIdx.x & 16;
    float half[kHalf];
#pragma unroll
    for (int k = 0; k < kHalf; ++k) {
      const float give = upper ? v[k] : v[k + kHalf];
      half[k] = (upper ? v[k + kHalf] : v[k]) + __shfl_xor_sync(0xffffffffu, give, 16);
    }
    if constexpr (N == 2) {
      half[0] = group_sum<16>(half[0]);
    } else {
      static_assert(N == 4, "");
      const bool high = threadIdx.x & 8;
      const float give = high ? half[0] : half[1];
      half[0] = (high ? half[1] : half[0]) + __shfl_xor_sync(0xffffffffu, give, 8);
      half[0] = group_sum<8>(half[0]);
    }
    v[0] = half[0];
  }
}
// N sums at once, in all threads of the row; `red`: [warps of the row][N], 16-byte aligned.
template <int TPR, int BLOCK, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red) {
  lane_sums<N, (TPR < 32 ? TPR : 32)>(v);
  if constexpr (TPR == 32 && N > 1) {
#pragma unroll
    for (int k = N - 1; k >= 0; --k) v[k] = __shfl_sync(0xffffffffu, v[0], k * (32 / N));
  }
  if constexpr (TPR > 32) {
    constexpr int kWarps = TPR / 32;
    if (threadIdx.x % (32 / N) == 0) red[threadIdx.x % TPR / (32 / N)] = v[0];
    group_barrier<TPR, BLOCK>();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.f;
    if constexpr (kWarps * N <= 8) {
#pragma unroll
      for (int w = 0; w < kWarps * N; w += 2) {
        const float2 s = *reinterpret_cast<const float2*>(red + w);
        v[w % N] += s.x;
        v[(w + 1) % N] += s.y;
      }
    } else {                               // a word per lane, and the warps' words of a number are added by shuffles
      const int lane = threadIdx.x % 32;
      float s = lane < kWarps * N ? red[lane] : 0.f;
      if constexpr (kWarps * N > 32) s += red[lane + 32];
#pragma unroll
      for (int o = N; o < (kWarps * N < 32 ? kWarps * N : 32); o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, s, k);
    }
  }
}

}  // namespace prm
