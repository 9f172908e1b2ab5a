// Rows streamed through shared memory by bulk asynchronous copies, for the row operators on large
// matrices: one persistent CTA per SM, whose warps form groups of W that walk over rows of their
// own.  A group's ring holds up to kRingStages rows of each of its input matrices.  A warp that
// is done with its part of a row says so on the stage's barrier; one more warp, a lane per group,
// sends for the row that takes the stage when all warps of the group have.  Bytes in flight are then
// set by the ring (up to 200 KB per SM), not by how many loads threads hold in registers between
// barriers.  (With a thread of the group sending, each row cost its group about 500 cycles more.)
//
// Waits are bounded.  A thread whose wait ran out sets the status word and touches no data any
// more, but keeps arriving at its group's barriers, so that nobody waits for it.
#pragma once

#include "async_copy.cuh"
#include "q8.cuh"

namespace prm {

constexpr int kRingStages = 6;
constexpr size_t kRingBytes = 200 * 1024;

// Warps of a persistent CTA that work on rows: a thread holds up to 32 elements of a row of each matrix.
template <typename IO>
constexpr int kRingWarps = sizeof(IO) == 2 ? 16 : 8;
template <typename IO>
constexpr int kRingThreads = kRingWarps<IO> * 32 + 32;

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
      ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
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
template <typename IO, int W, int ARR>
struct RingBlock {
  static constexpr int kGroups = kRingWarps<IO> / W;
  uint64_t full[kGroups][kRingStages];    // the copies of a row have landed
  uint64_t empty[kGroups][kRingStages];   // W warps are done with the row
  alignas(16) float red[kGroups][2][32];
  int abort_word;
};
template <typename IO, int W, int ARR>
__device__ __forceinline__ RingBlock<IO, W, ARR>& ring_block() {
  __shared__ RingBlock<IO, W, ARR> b;
  return b;
}

// One group's ring over ARR matrices of the same number of rows.  The group's row number i (0, 1,
// ..., n - 1) is row first + i * step.
template <typename IO, int W, int ARR>
struct RowRing {
  RingBlock<IO, W, ARR>& b;
  const IO* src[ARR];
  int64_t ld[ARR];
  int first, step, n;     // rows (below 2^31)
  uint8_t* base;          // [stages][ARR][row_bytes]
  uint32_t row_bytes;
  int stages, group, stage;
  uint32_t phase;
  int laps, last;         // of the walk back: (n - 1) / stages and its remainder
  bool producer, ok;
  int* status;

  __device__ __forceinline__ RowRing(RingBlock<IO, W, ARR>& block, const void* const* srcs, const int64_t* lds,
                                     int rows, int cols, int n_stages, int* status_word)
      : b(block), stages(n_stages), stage(0), phase(0), ok(true), status(status_word) {
    constexpr int kGroups = kRingWarps<IO> / W;
    producer = threadIdx.x >= kRingWarps<IO> * 32;
    group = producer ? threadIdx.x - kRingWarps<IO> * 32 : threadIdx.x / (W * 32);   // a lane per group
#pragma unroll
    for (int k = 0; k < ARR; ++k) {
      src[k] = reinterpret_cast<const IO*>(srcs[k]);
      ld[k] = lds[k];
    }
    row_bytes = (uint32_t)cols * sizeof(IO);
    base = ring_memory() + (size_t)group * stages * ARR * row_bytes;
    place(blockIdx.x, gridDim.x, rows);
  }
  // The rows of a block that is number `line` of `lines`.
  __device__ __forceinline__ void place(int line, int lines, int rows) {
    constexpr int kGroups = kRingWarps<IO> / W;
    first = line * kGroups + group;
    step = lines * kGroups;
    n = group < kGroups && first < rows ? (rows - first - 1) / step + 1 : 0;
  }
  __device__ __forceinline__ int64_t row(int i) const { return first + (int64_t)i * step; }
  __device__ __forceinline__ const IO* at(int k) const {
    return reinterpret_cast<const IO*>(base + ((size_t)stage * ARR + k) * row_bytes);
  }
  __device__ __forceinline__ void fetch(int i, int s) const {
    const int64_t r = row(i);
    mbar_expect_tx(&b.full[group][s], ARR * row_bytes);
#pragma unroll
    for (int k = 0; k < ARR; ++k)
      bulk_load(base + ((size_t)s * ARR + k) * row_bytes, src[k] + r * ld[k], row_bytes, &b.full[group][s]);
  }
  // All threads of the block, once.
  __device__ __forceinline__ void start() {
    constexpr int kBars = (kRingWarps<IO> / W) * kRingStages;
    if (threadIdx.x < kBars) {
      mbar_init(&b.full[0][0] + threadIdx.x, 1);
      mbar_init(&b.empty[0][0] + threadIdx.x, W);
    }
    if (threadIdx.x == 0) b.abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  }
  // The producer's lanes, each for its group: rows 0 .. n - 1.  No lane waits for another's row.
  __device__ __forceinline__ void serve() {
    int i = 0;
    Patience p;
    while (__any_sync(0xffffffffu, ok && i < n)) {
      if (ok && i < n) {
        if (i < stages || mbar_test(&b.empty[group][stage], phase ^ 1)) {
          fetch(i, stage);
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
  // The current row has landed.
  __device__ __forceinline__ bool wait() {
    ok = ok && mbar_wait(&b.full[group][stage], phase, &b.abort_word, status);
    return ok;
  }
  // This warp is done with the current row.
  __device__ __forceinline__ void release() const {
    __syncwarp();
    if ((threadIdx.x & 31) == 0 && ok) mbar_arrive(&b.empty[group][stage]);
  }
  // Barrier of the group (named barriers 1 .. 8; a group of one warp needs none).
  __device__ __forceinline__ void sync() const {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
  }
  // A second walk over the same rows, last row first.  The last `stages` rows are still in the ring;
  // the others are sent for again as their stages fall free.  Between the two walks lies a barrier of
  // the block.  wait_back(i) / release() / retreat() go with i = n - 1, ..., 0.
  __device__ __forceinline__ void turn_back() {
    laps = n > 0 ? (n - 1) / stages : 0;
    last = stage = n > 0 ? (n - 1) % stages : 0;
    phase = 0;
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
    if (stage == last) ++phase;             // laps of the walk back
  }
  __device__ __forceinline__ void serve_back() {
    int i = n - 1 - stages;                 // row i takes the stage of row i + stages
    phase = 1;
    Patience p;
    while (__any_sync(0xffffffffu, ok && i >= 0)) {
      if (ok && i >= 0) {
        if (mbar_test(&b.empty[group][stage], (fills() - 1) & 1u)) {
          fetch(i, stage);
          --i;
          retreat();
          p = Patience();
        } else {
          lose(p);
        }
      }
    }
  }
  // Reductions over the group; the words of row i and row i + 1 lie apart and are read in pieces.
  static constexpr int kPiece = W >= 4 ? 4 : 2;
  struct Words {
    float v[kPiece];
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
  };
  static __device__ __forceinline__ Words words(const float* p) {
    Words w;
    if constexpr (kPiece == 4) {
      const float4 f = *reinterpret_cast<const float4*>(p);
      w.v[0] = f.x; w.v[1] = f.y; w.v[2] = f.z; w.v[3] = f.w;
    } else {
      const float2 f = *reinterpret_cast<const float2*>(p);
      w.v[0] = f.x; w.v[1] = f.y;
    }
    return w;
  }
  __device__ __forceinline__ void sum2(int i, float& p, float& q) const {
    p = warp_sum(p);
    q = warp_sum(q);
    if constexpr (W > 1) {
      float* red = b.red[group][i & 1];
      const int warp = (threadIdx.x >> 5) % W;
      if ((threadIdx.x & 31) == 0) {
        red[warp] = p;
        red[16 + warp] = q;
      }
      sync();
      p = q = 0.f;
#pragma unroll
      for (int k = 0; k < W; k += kPiece) {
        const auto u = words(red + k), v = words(red + 16 + k);
#pragma unroll
        for (int e = 0; e < kPiece; ++e) {
          p += u[e];
          q += v[e];
        }
      }
    }
  }
  __device__ __forceinline__ void max_top(int i, float& top) const {
    top = warp_top(top);
    if constexpr (W > 1) {
      float* red = b.red[group][i & 1];
      if ((threadIdx.x & 31) == 0) red[(threadIdx.x >> 5) % W] = top;
      sync();
      top = 0.f;
#pragma unroll
      for (int k = 0; k < W; k += kPiece) {
        const auto v = words(red + k);
#pragma unroll
        for (int e = 0; e < kPiece; e += 2) top = max_abs(top, make_float2(v[e], v[e + 1]));
      }
    }
  }
  __device__ __forceinline__ void sum_top(int i, float& p, float& top) const {
    p = warp_sum(p);
    top = warp_top(top);
    if constexpr (W > 1) {
      float* red = b.red[group][i & 1];
      const int warp = (threadIdx.x >> 5) % W;
      if ((threadIdx.x & 31) == 0) {
        red[warp] = p;
        red[16 + warp] = top;
      }
      sync();
      p = top = 0.f;
#pragma unroll
      for (int k = 0; k < W; k += kPiece) {
        const auto u = words(red + k), v = words(red + 16 + k);
#pragma unroll
        for (int e = 0; e < kPiece; e += 2) {
          p += u[e] + u[e + 1];
          top = max_abs(top, make_float2(v[e], v[e + 1]));
        }
      }
    }
  }
  // Copies in flight land before the CTA's memory goes (only after a wait that ran out are there any).
  __device__ __forceinline__ void finish() const {
    if (*(volatile int*)&b.abort_word && producer) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 1000000ull) {
      }
    }
  }
};

// ------------------------------------------------------------------ host side

// The status word that prm_q8_status reads, on the current device (null if it has none).
int* q8_status_word();

constexpr int kRingBlocks = 148;     // one CTA per SM

// From here on streaming is faster than one row per block.
constexpr int64_t kRingElements = 1 << 22;
inline bool ring_worth(int64_t rows, int cols) { return cols >= 512 && cols <= 8192 && rows * cols >= kRingElements; }
inline int ring_blocks(int64_t rows, int groups) { return (int)std::min<int64_t>(kRingBlocks, (rows + groups - 1) / groups); }

// One CTA per SM; `extra` bytes are what the kernel wants of the ring's memory after the last row.
template <typename IO, int W, bool COOPERATIVE = false, typename A>
int launch_ring(void (*kernel)(A, int, int*), int arrays, PerDeviceOnce& once, int64_t rows, int cols, size_t extra, cudaStream_t stream,
                A a) {
  constexpr int kGroups = kRingWarps<IO> / W;
  int dev;
  if (once.need(&dev)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes) != cudaSuccess)
      return PRM_ERR_CUDA;
    once.mark(dev);
  }
  int* status = q8_status_word();
  const size_t row = (size_t)cols * sizeof(IO) * arrays * kGroups;
  const int stages = (int)std::min<size_t>(kRingStages, kRingBytes / row);
  if (!status || stages < 1 || extra > kRingBytes) return PRM_ERR_CUDA;
  const unsigned blocks = (unsigned)ring_blocks(rows, kGroups);
  const size_t smem = std::max(extra, row * stages);
  cudaError_t e;
  if constexpr (COOPERATIVE) {
    int n = stages;
    void* args[3] = {&a, &n, &status};
    e = cudaLaunchCooperativeKernel((const void*)kernel, dim3(blocks), dim3(kRingThreads<IO>), args, smem, stream);
  } else {
    e = launch_after(kernel, blocks, kRingThreads<IO>, smem, stream, 0, a, stages, status);
  }
  return e == cudaSuccess ? PRM_OK : PRM_ERR_CUDA;
}

}  // namespace prm
