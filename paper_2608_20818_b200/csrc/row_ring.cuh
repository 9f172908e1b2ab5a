// Rows streamed through shared memory by bulk asynchronous copies, for the row operators on large
// matrices: one persistent CTA per SM, whose 16 warps form groups of W that walk over sets of R
// neighbouring rows of their own.  A group's ring holds up to kRingStages sets of each of its input
// matrices.  A warp that is done with its part of a set says so on the stage's barrier; one more warp,
// a lane per group, sends for the set that takes the stage when all warps of the group have.  Bytes in
// flight are then set by the ring (up to 200 KB per SM), not by how many loads threads hold in
// registers between barriers.
//
// What bounds such a kernel next to HBM is instructions per element: the barrier, the addressing and
// (with R = 2) the weights or factors that a thread holds for its columns are shared by the 32 elements
// that it has of a set, as one row of four octs or as two rows of two.  Which of the two is faster was
// measured for each kernel: narrow rows and sums over rows gain by two rows, wide rows lose by a
// group that is the whole CTA.
//
// Waits are bounded.  A thread whose wait ran out sets the status word and touches no data any
// more, but keeps arriving at its group's barriers, so that nobody waits for it.
#pragma once

#include <type_traits>

#include "async_copy.cuh"
#include "q8.cuh"
#include "q8_plan.h"

namespace prm {

constexpr int kRingStages = 6;
constexpr size_t kRingBytes = 200 * 1024;
constexpr int kRingWarps = 16;                        // that work on rows
constexpr int kRingThreads = kRingWarps * 32 + 32;    // and the producer

// Rows per set of the kernels that take two: one where the elements are 32 bits wide, for the registers.
template <typename IO>
constexpr int kRingRows = sizeof(IO) == 2 ? 2 : 1;

// `policy`: how long the L2 should hold the lines (evict_first / evict_last below).
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
      ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}
__device__ __forceinline__ uint64_t evict_first() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t evict_last() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
// Whether a phase is complete, without the suspension that mbarrier.try_wait may put in: the producer's
// lanes wait for barriers of their own and none may hold up the others.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint8_t* ring_memory() {
  extern __shared__ __align__(128) uint8_t ring_mem[];
  return ring_mem;
}

// The static shared memory of a CTA's rings.
template <int W, int R>
struct RingBlock {
  static constexpr int kGroups = kRingWarps / W;
  uint64_t full[kGroups][kRingStages];    // the copies of a set have landed
  uint64_t empty[kGroups][kRingStages];   // W warps are done with the set
  alignas(16) float red[kGroups][2][R][2][16];
  int abort_word;
};
template <int W, int R>
__device__ __forceinline__ RingBlock<W, R>& ring_block() {
  __shared__ RingBlock<W, R> b;
  return b;
}

// One group's ring over ARR matrices of the same number of rows.  The group's set number i (0, 1,
// ..., n - 1) are the rows (first + i * step) * R and up to R - 1 after it.
template <typename IO, int W, int R, int ARR>
struct RowRing {
  static constexpr int kGroups = kRingWarps / W;
  RingBlock<W, R>& b;
  const IO* src[ARR];
  int64_t ld[ARR];
  int rows, first, step, n;
  uint8_t* base;          // [stages][R][ARR][row_bytes]
  uint32_t row_bytes;
  int stages, group, stage;
  uint32_t phase;
  int laps, last;         // of the walk back: (n - 1) / stages and its remainder
  bool producer, ok;
  int* status;

  __device__ __forceinline__ RowRing(RingBlock<W, R>& block, const void* const* srcs, const int64_t* lds, int64_t n_rows,
                                     int cols, int n_stages, int* status_word)
      : b(block), rows((int)n_rows), stages(n_stages), stage(0), phase(0), ok(true), status(status_word) {
    producer = threadIdx.x >= kRingWarps * 32;
    group = producer ? threadIdx.x - kRingWarps * 32 : threadIdx.x / (W * 32);   // a lane per group
#pragma unroll
    for (int k = 0; k < ARR; ++k) {
      src[k] = reinterpret_cast<const IO*>(srcs[k]);
      ld[k] = lds[k];
    }
    row_bytes = (uint32_t)cols * sizeof(IO);
    base = ring_memory() + (size_t)group * stages * R * ARR * row_bytes;
    place(blockIdx.x, gridDim.x);
  }
  // The sets of a block that is number `line` of `lines`.
  __device__ __forceinline__ void place(int line, int lines) {
    const int sets = (rows - 1) / R + 1;
    first = line * kGroups + group;
    step = lines * kGroups;
    n = group < kGroups && first < sets ? (sets - first - 1) / step + 1 : 0;
  }
  __device__ __forceinline__ int64_t row(int i) const { return ((int64_t)i * step + first) * R; }
  // Rows of set i: R, but for the last one.
  __device__ __forceinline__ int height(int i) const { return R == 1 ? 1 : (int)min((int64_t)R, rows - row(i)); }
  // Row r of matrix k of the current set.
  __device__ __forceinline__ const IO* at(int r, int k) const {
    return reinterpret_cast<const IO*>(base + (uint32_t)((stage * R + r) * ARR + k) * row_bytes);
  }
  __device__ __forceinline__ void fetch(int i, int s, uint64_t policy) const {
    const int h = height(i);
    mbar_expect_tx(&b.full[group][s], (uint32_t)(h * ARR) * row_bytes);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r < h) {
#pragma unroll
        for (int k = 0; k < ARR; ++k)
          bulk_load(base + (uint32_t)((s * R + r) * ARR + k) * row_bytes, src[k] + (row(i) + r) * ld[k], row_bytes,
                    &b.full[group][s], policy);
      }
    }
  }
  // All threads of the block, once.
  __device__ __forceinline__ void start() {
    constexpr int kBars = kGroups * kRingStages;
    if (threadIdx.x < kBars) {
      mbar_init(&b.full[0][0] + threadIdx.x, 1);
      mbar_init(&b.empty[0][0] + threadIdx.x, W);
    }
    if (threadIdx.x == 0) b.abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  }
  // The producer's lanes, each for its group: sets 0 .. n - 1.  No lane waits for another's set.  Sets
  // from `keep` on will be read again and stay in the L2; those before them make room.
  __device__ __forceinline__ void serve(int keep = 0x7fffffff) {
    const uint64_t once = evict_first(), again = evict_last();
    int i = 0;
    Patience p;
    while (__any_sync(0xffffffffu, ok && i < n)) {
      if (ok && i < n) {
        if (i < stages || mbar_test(&b.empty[group][stage], phase ^ 1)) {
          fetch(i, stage, i < keep ? once : again);
          ++i;
          advance();
          p = Patience();
        } else {
          lose(p);
        }
      }
    }
  }
  __device__ __forceinline__ void advance() {
    if (++stage == stages) {
      stage = 0;
      phase ^= 1;
    }
  }
  // One more poll without success: every 256th looks at the clock and at the others.
  struct Patience {
    uint32_t polls = 0;
    uint64_t t0 = 0;
  };
  __device__ __forceinline__ void lose(Patience& p) {
    if ((++p.polls & 255u) != 0) return;
    const uint64_t now = global_ns();
    if (p.t0 == 0) p.t0 = now;
    if (*(volatile int*)&b.abort_word) ok = false;
    if (now - p.t0 > kWaitLimitNs) {
      ok = false;
      *(volatile int*)&b.abort_word = 1;
      atomicOr(status, kStatusTimeout);
    }
  }
  // The current set has landed.
  __device__ __forceinline__ bool wait() {
    ok = ok && mbar_wait(&b.full[group][stage], phase, &b.abort_word, status);
    return ok;
  }
  // This warp is done with the current set.
  __device__ __forceinline__ void release() const {
    __syncwarp();
    if ((threadIdx.x & 31) == 0 && ok) mbar_arrive(&b.empty[group][stage]);
  }
  // Barrier of the group (named barriers 1 .. 8; a group of one warp needs none).
  __device__ __forceinline__ void sync() const {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
  }
  // A second walk over the same sets, last one first.  The last `stages` sets are still in the ring;
  // the others are sent for again as their stages fall free.  Between the two walks lies a barrier of
  // the block.  wait_back(i) / release() / retreat() go with i = n - 1, ..., 0.
  __device__ __forceinline__ void turn_back() {
    laps = n > 0 ? (n - 1) / stages : 0;
    last = stage = n > 0 ? (n - 1) % stages : 0;
    phase = 0;                              // laps of the walk back
  }
  // Copies into (and releases of) the current stage on the way out, plus the laps since.
  __device__ __forceinline__ uint32_t fills() const { return (uint32_t)laps + (stage <= last ? 1u : 0u) + phase; }
  __device__ __forceinline__ bool wait_back(int i) {
    if (i < n - stages)
      ok = ok && mbar_wait(&b.full[group][stage], (fills() - 1) & 1u, &b.abort_word, status);
    return ok;
  }
  __device__ __forceinline__ void retreat() {
    if (stage == 0) stage = stages;
    --stage;
    if (stage == last) ++phase;
  }
  __device__ __forceinline__ void serve_back() {
    const uint64_t once = evict_first();
    int i = n - 1 - stages;                 // set i takes the stage of set i + stages
    phase = 1;
    Patience p;
    while (__any_sync(0xffffffffu, ok && i >= 0)) {
      if (ok && i >= 0) {
        if (mbar_test(&b.empty[group][stage], (fills() - 1) & 1u)) {
          fetch(i, stage, once);
          --i;
          retreat();
          p = Patience();
        } else {
          lose(p);
        }
      }
    }
  }
  // Reductions over the group, R rows with one barrier.  The words of set i and set i + 1 lie apart.
  // SUMS: two sums, else one largest magnitude (q).
  static constexpr int kPiece = W >= 4 ? 4 : 2;
  template <bool SUMS>
  __device__ __forceinline__ void reduce(int i, float (&p)[R], float (&q)[R]) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if constexpr (SUMS) p[r] = warp_sum(p[r]);
      q[r] = SUMS ? warp_sum(q[r]) : group_top(q[r]);
    }
    if constexpr (W > 1) {
      float(*red)[2][16] = b.red[group][i & 1];
      const int warp = (threadIdx.x >> 5) % W;
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if constexpr (SUMS) red[r][0][warp] = p[r];
          red[r][1][warp] = q[r];
        }
      }
      sync();
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (SUMS) p[r] = 0.f;
        q[r] = 0.f;
#pragma unroll
        for (int k = 0; k < W; k += kPiece) {
          float u[kPiece], v[kPiece];
          if constexpr (SUMS) words(red[r][0] + k, u);
          words(red[r][1] + k, v);
#pragma unroll
          for (int e = 0; e < kPiece; e += 2) {
            if constexpr (SUMS) p[r] += u[e] + u[e + 1];
            if constexpr (SUMS) q[r] += v[e] + v[e + 1];
            else q[r] = max_abs(q[r], make_float2(v[e], v[e + 1]));
          }
        }
      }
    }
  }
  static __device__ __forceinline__ void words(const float* p, float (&w)[kPiece]) {
    if constexpr (kPiece == 4) {
      const float4 f = *reinterpret_cast<const float4*>(p);
      w[0] = f.x; w[1] = f.y; w[2] = f.z; w[3] = f.w;
    } else {
      const float2 f = *reinterpret_cast<const float2*>(p);
      w[0] = f.x; w[1] = f.y;
    }
  }
  // All threads of the block, after the last set.  Copies in flight land before the CTA's memory goes: there
  // are any only after a wait that ran out, which may be a consumer's after the producer's last copy.
  __device__ __forceinline__ void finish() const {
    __syncthreads();
    if (*(volatile int*)&b.abort_word) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 1000000ull) {
      }
    }
  }
};

// ------------------------------------------------------------------ host side

// The status word that prm_q8_status reads, on the current device (null if it has none).
int* q8_status_word();
// SMs of the current device that persistent and cooperative launches use (0: an error).
int q8_sms();

// Calls f with the number of warps to a row of up to 8192 elements, two octs per thread.
template <typename F>
int with_ring_warps(int cols, F f) {
  if (cols <= 512) return f(std::integral_constant<int, 1>());
  if (cols <= 1024) return f(std::integral_constant<int, 2>());
  if (cols <= 2048) return f(std::integral_constant<int, 4>());
  if (cols <= 4096) return f(std::integral_constant<int, 8>());
  return f(std::integral_constant<int, 16>());
}

// Cooperative launch of kernel(a, stages, status): `set_bytes` of ring per stage and CTA, then `tail` bytes
// that the kernel uses beside the ring.
template <typename A>
int launch_ring(void (*kernel)(A, int, int*), PerDeviceOnce& once, unsigned blocks, size_t set_bytes, size_t tail,
                cudaStream_t stream, A a) {
  int dev;
  if (once.need(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
    if (e != cudaSuccess) return q8_code(e);
    once.mark(dev);
  }
  int* status = q8_status_word();
  if (tail > kRingBytes) return PRM_ERR_CUDA;
  int stages = (int)std::min<size_t>(kRingStages, (kRingBytes - tail) / set_bytes);
  if (!status || stages < 1) return PRM_ERR_CUDA;
  void* args[3] = {&a, &stages, &status};
  return q8_code(cudaLaunchCooperativeKernel((const void*)kernel, dim3(blocks), dim3(kRingThreads), args,
                                             set_bytes * stages + tail, stream));
}

}  // namespace prm
