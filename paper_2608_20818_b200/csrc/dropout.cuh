// Dropout from a counter-based generator: whether an element stays is a function of its row, its column and
// the number of the draw, so that no mask is stored and the gradient draws the same one again.
//
//   keep(i, j):  word j % 4 of Philox4x32-10 at the counter (j / 4, i, low s, high s) under the key `seed`
//                >= p 2^32,    s = offset + *counter
//   out(i, j) = keep ? x(i, j) * (1 / (1 - p)) : 0
//
// Philox4x32-10 is the generator of Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
// 1, 2, 3" (SC 2011): ten rounds of two 32 x 32 -> 64 bit products, whose halves change places, under a key
// that advances by a constant (the rounds' keys come with the kernel's arguments: computed by every thread they
// cost 8192 x 8192 bf16 elements 9 us more).  Four elements share one evaluation: 18 to 20 products of four
// cycles of an SM's quarter and 20 exclusive ors of two, alone 0.66 cycles of an SM, 39 us for 8192 x 8192 elements (memory
// alone: 41 us); a product as one half from double precision and one from 32-bit integers takes 0.9.
#pragma once

#include <cmath>

#include "q8.cuh"

namespace prm {

// As the kernels take it.  counter may be null (0).
struct Drop {
  uint32_t threshold = 0;                  // a word below it drops its element
  float scale = 1.f;
  uint2 key[10] = {};                      // of each round
  uint64_t offset = 0;
  const uint64_t* counter = nullptr;
};

inline bool drop_ok(double p) { return p >= 0.0 && p < 1.0; }      // false for a NaN too
inline Drop make_drop(double p, uint64_t seed, uint64_t offset, const uint64_t* counter) {
  Drop d;
  // p > 0 has a threshold: that there is one is what the kernels go by
  if (p > 0.0) d.threshold = (uint32_t)std::min(std::max(std::nearbyint(p * 4294967296.0), 1.0), 4294967295.0);
  d.scale = (float)(1.0 / (1.0 - p));
  for (uint32_t r = 0; r < 10; ++r)
    d.key[r] = make_uint2((uint32_t)seed + r * 0x9E3779B9u, (uint32_t)(seed >> 32) + r * 0xBB67AE85u);
  d.offset = offset;
  d.counter = counter;
  return d;
}

__device__ __forceinline__ uint64_t drop_number(const Drop& d) { return d.offset + (d.counter ? *d.counter : 0); }

__device__ __forceinline__ uint4 philox(uint4 c, const uint2 (&key)[10]) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ key[r].x, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ key[r].y, (uint32_t)a);
  }
  return c;
}
// The words of the elements 4 quad .. 4 quad + 3 of a row.
__device__ __forceinline__ uint4 drop_words(const Drop& d, uint64_t number, uint32_t row, uint32_t quad) {
  return philox(make_uint4(quad, row, (uint32_t)number, (uint32_t)(number >> 32)), d.key);
}
// The product is rounded by itself (nothing is fused through the choice).
__device__ __forceinline__ float dropped(const Drop& d, uint32_t word, float v) {
  return word >= d.threshold ? __fmul_rn(v, d.scale) : 0.f;
}

// The oct of elements first .. first + 7; EVEN: first is a multiple of 4.  Elements outside the row get any value.
template <bool EVEN>
__device__ __forceinline__ void drop_oct(const Drop& d, uint64_t number, uint32_t row, int first, float2 (&v)[4]) {
  const int quad = first >> 2;
  const uint4 a = drop_words(d, number, row, (uint32_t)quad), b = drop_words(d, number, row, (uint32_t)quad + 1);
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if constexpr (!EVEN) {
    const int off = first & 3;             // alike for all octs of a row
    if (off) {
      const uint4 c = drop_words(d, number, row, (uint32_t)quad + 2);
      const uint32_t more[3] = {c.x, c.y, c.z};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t one = k + 1 < 8 ? w[k + 1] : more[k - 7], two = k + 2 < 8 ? w[k + 2] : more[k - 6],
                       three = k + 3 < 8 ? w[k + 3] : more[k - 5];
        w[k] = off == 1 ? one : off == 2 ? two : three;      // ascending k: what is read has not been changed
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 scaled = mul2(v[k], make_float2(d.scale, d.scale));
    v[k] = make_float2(w[2 * k] >= d.threshold ? scaled.x : 0.f, w[2 * k + 1] >= d.threshold ? scaled.y : 0.f);
  }
}

}  // namespace prm
