// The 8-bit product for shapes that fill the GPU with 256 x 256 tiles: persistent CTA pairs on
// tcgen05.mma.cta_group::2.
//
// A pair computes out[m0 .. m0+255, n0 .. n0+255].  CTA r of the pair holds rows m0 + 128 r .. + 127 of
// a (the matrix instruction's M, and those lanes of the accumulator) and 128 of the 256 columns of b.
//
//   warp 0      TMA producer: per stage 256 k of both operands (64 KB), 128-byte swizzle, no multicast;
//               the copies of both CTAs count on the leader's barrier.  Three stages
//   warp 1      tcgen05.mma issuer (one lane of the leader); owns its CTA's tensor memory
//   warps 2..9  epilogue: two warps per lane quadrant, half of the 256 columns each.  A thread scales
//               64 bytes of a row at a time in pairs of values; they pass through 2 KB of shared memory
//               per warp, from which four neighbouring lanes store a row's 64 bytes (rows or widths
//               that are not 16-byte aligned: element by element).  Straight from registers, with
//               the lanes along n, the same tile took 6,000 cycles instead of 4,900
// Two accumulators of 256 columns let the epilogue of a tile run under the next tile's main loop.
// Every barrier wait is bounded; one that runs out sets the status word, the pair drains and leaves.
#include "q8_matmul.cuh"

namespace prm {
namespace {

constexpr int kTile = 256;                       // tile edge, both ways
constexpr int kSub = 2;                          // k-blocks per stage
constexpr int kStages = 3;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 32 * (2 + kEpiWarps);
constexpr uint32_t kBoxBytes = 128 * kBlockK;    // 128 rows of one k-block
constexpr uint32_t kStageBytes = 2 * kSub * kBoxBytes;
constexpr uint32_t kPatchBytes = 32 * 64;        // a warp's 32 rows of 64 bytes on their way out
constexpr uint32_t kEpiBytes = kEpiWarps * (kPatchBytes + 128 * 4);     // and its 128 column scales
constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + kEpiBytes;

// Load whose completion is counted on the pair leader's barrier (a shared::cluster address).
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* map, uint32_t bar_cluster, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_u32(dst)), "l"((uint64_t)map), "r"(bar_cluster), "r"(x), "r"(y)
      : "memory");
}
template <bool INT8>
__device__ __forceinline__ void umma_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                          uint32_t accumulate) {
  if constexpr (INT8) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
  }
}
// Arrives, once all matrix instructions issued so far are done, on the barrier at this
// shared-memory offset in both CTAs of the pair (a barrier arrival, not a load).
__device__ __forceinline__ void umma_commit_both(uint32_t bar) {
  const uint16_t mask = 3;
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"(mask)
               : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}

struct PairArgs {
  MatmulArgs c;
  int m_tiles, n_tiles, tiles;
  int band;               // m-tiles that are walked through together
};

// Order of the tiles: bands of `band` m-tiles, in a band n by n, m-tiles fastest.  Pairs that run at the
// same time then share the band's rows of a and a few columns' worth of b.
__device__ __forceinline__ void tile_origin(const PairArgs& a, int t, int& m0, int& n0) {
  const int per = a.band * a.n_tiles, first = t / per * a.band, rest = t % per;
  const int height = min(a.band, a.m_tiles - first);
  m0 = (first + rest % height) * kTile;
  n0 = rest / height * kTile;
}

// One warp's 32 rows by 128 columns of a finished accumulator: lane = row, `taddr` its first column.
template <bool INT8, typename OUT>
__device__ __forceinline__ void store_tile(const PairArgs& a, uint32_t taddr, float sa, const float* sb, uint8_t* patch,
                                           int m0, int n0, int rows) {
  constexpr int kCols = 64 / sizeof(OUT);                 // per piece
  const int lane = threadIdx.x & 31;
  OUT* out = reinterpret_cast<OUT*>(a.c.out) + (int64_t)m0 * a.c.ld_out + n0;
  const bool vec = ((uintptr_t)out & 15) == 0 && (a.c.ld_out * (int64_t)sizeof(OUT)) % 16 == 0;
  // 16-byte chunk c of row r lies where neither writing rows nor reading them back meets a bank twice.
  auto at = [&](int r, int c) { return reinterpret_cast<uint4*>(patch + (r >> 1) * 128 + (r & 1) * 64 + ((c ^ ((r >> 1) & 3)) << 4)); };
  const float2 sa2 = make_float2(sa, sa);
#pragma unroll 1
  for (int k = 0; k < 128 / 32; ++k) {
    uint32_t r[32];
    tmem_ld32(taddr + k * 32, r);
    tmem_wait_ld();
#pragma unroll
    for (int piece = 0; piece < 32 / kCols; ++piece) {
      const int n = n0 + k * 32 + piece * kCols, wide = min(kCols, a.c.n - n);
      if (wide <= 0) break;
      uint4 w[4];
#pragma unroll
      for (int c = 0; c < kCols / 4; ++c) {
        const float4 f = *reinterpret_cast<const float4*>(sb + k * 32 + piece * kCols + c * 4);
        const uint32_t* q = r + piece * kCols + c * 4;
        auto value = [&](int e) { return INT8 ? (float)(int)q[e] : __uint_as_float(q[e]); };
        const float2 u = mul2(mul2(make_float2(value(0), value(1)), sa2), make_float2(f.x, f.y));
        const float2 v = mul2(mul2(make_float2(value(2), value(3)), sa2), make_float2(f.z, f.w));
        uint32_t* o = reinterpret_cast<uint32_t*>(w);
        if constexpr (sizeof(OUT) == 2) {
          o[c * 2] = pair_to_bf16(u);
          o[c * 2 + 1] = pair_to_bf16(v);
        } else {
          o[c * 4] = __float_as_uint(u.x);
          o[c * 4 + 1] = __float_as_uint(u.y);
          o[c * 4 + 2] = __float_as_uint(v.x);
          o[c * 4 + 3] = __float_as_uint(v.y);
        }
      }
      __syncwarp();                                       // the piece before has been read
#pragma unroll
      for (int c = 0; c < 4; ++c) *at(lane, c) = w[c];
      __syncwarp();
      OUT* to = out + k * 32 + piece * kCols;
      if (vec && wide == kCols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = i * 8 + (lane >> 2);
          const uint4 x = *at(row, lane & 3);
          if (row < rows) *reinterpret_cast<uint4*>(to + row * a.c.ld_out + (lane & 3) * (16 / sizeof(OUT))) = x;
        }
      } else {
#pragma unroll 4
        for (int row = 0; row < rows; ++row) {
          const int c = lane * (int)sizeof(OUT);
          if (lane < wide)
            to[row * a.c.ld_out + lane] =
                *reinterpret_cast<const OUT*>(reinterpret_cast<const uint8_t*>(at(row, (c >> 4) & 3)) + (c & 15));
        }
      }
    }
  }
}

template <bool INT8, bool P_MN, bool Q_MN>
__global__ void __launch_bounds__(kThreads, 1)
matmul_q8_pair_kernel(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q,
                      const PairArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kStages], empty[kStages], tfull[2], tempty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  volatile int* abort_flag = &abort_word;
  int* status = a.c.status;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int stages_k = (a.c.kblocks + kSub - 1) / kSub;          // stages per tile

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], 2 * kEpiWarps);
    }
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tcgen05_before_sync();
  __syncthreads();
  cluster_barrier();                             // the peer's barriers are initialised too
  tcgen05_after_sync();
  const uint32_t tmem = tmem_slot;
  grid_wait();
  grid_trigger();                                // not before the tensor memory is this kernel's

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      const uint32_t lead_full = cluster_map(smem_u32(&full[0]), 0);
      for (int t = pair; t < a.tiles && ok; t += pairs) {
        int m0, n0;
        tile_origin(a, t, m0, n0);
        m0 += (int)rank * 128;
        n0 += (int)rank * 128;
        for (int kt = 0; kt < stages_k; ++kt, ++it) {
          const int s = it % kStages;
          if (!mbar_wait(&empty[s], ((it / kStages) & 1) ^ 1, abort_flag, status)) { ok = false; break; }
          uint8_t* sp = smem + (size_t)s * kStageBytes;
          uint8_t* sq = sp + kSub * kBoxBytes;
          const int subs = min(kSub, a.c.kblocks - kt * kSub);
          if (rank == 0) mbar_expect_tx(&full[s], (uint32_t)subs * 4 * kBoxBytes);   // both CTAs' bytes
          const uint32_t bar = lead_full + 8u * s;
#pragma unroll
          for (int j = 0; j < kSub; ++j) {
            if (j < subs) {
              const int k0 = (kt * kSub + j) * kBlockK;
              tma_load_pair(sp + j * kBoxBytes, &map_p, bar, P_MN ? m0 : k0, P_MN ? k0 : m0);
              tma_load_pair(sq + j * kBoxBytes, &map_q, bar, Q_MN ? n0 : k0, Q_MN ? k0 : n0);
            }
          }
        }
      }
      // Copies in flight must land before shared memory is released; the leader sees both CTAs'.
      if (rank == 0) {
        for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j) {
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(&full[j % kStages], (j / kStages) & 1) && global_ns() - t0 < 1000000ull) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = idesc_8bit(INT8, kTile, kTile, P_MN, Q_MN);
      constexpr uint32_t kStepP = P_MN ? 256 : 2, kStepQ = Q_MN ? 256 : 2;    // 32 k, in units of 16 bytes
      uint32_t it = 0, acc = 0;
      bool ok = true;
      const uint32_t smem0 = smem_u32(smem);
      for (int t = pair; t < a.tiles && ok; t += pairs, ++acc) {
        const uint32_t ab = acc & 1;
        if (!mbar_wait(&tempty[ab], ((acc >> 1) & 1) ^ 1, abort_flag, status)) break;
        tcgen05_after_sync();
        const uint32_t d = tmem + ab * kTile;
        for (int kt = 0; kt < stages_k; ++kt, ++it) {
          const int s = it % kStages;
          if (!mbar_wait(&full[s], (it / kStages) & 1, abort_flag, status)) { ok = false; break; }
          tcgen05_after_sync();
          const uint32_t sp = smem0 + (uint32_t)s * kStageBytes, sq = sp + kSub * kBoxBytes;
          const int subs = min(kSub, a.c.kblocks - kt * kSub);
#pragma unroll
          for (int j = 0; j < kSub; ++j) {
            if (j < subs) {
              const uint64_t dp = P_MN ? desc_mn_major(sp + j * kBoxBytes, kBoxBytes) : desc_k_major(sp + j * kBoxBytes);
              const uint64_t dq = Q_MN ? desc_mn_major(sq + j * kBoxBytes, kBoxBytes) : desc_k_major(sq + j * kBoxBytes);
#pragma unroll
              for (int i = 0; i < kBlockK / 32; ++i)
                umma_pair<INT8>(d, dp + kStepP * i, dq + kStepQ * i, idesc, (kt | j | i) != 0);
            }
          }
          umma_commit_both(smem_u32(&empty[s]));
        }
        if (ok) umma_commit_both(smem_u32(&tfull[ab]));
      }
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * 128);
    const uint32_t lead_tempty = cluster_map(smem_u32(&tempty[0]), 0);
    uint8_t* own = smem + (size_t)kStages * kStageBytes + (warp - 2) * (kPatchBytes + 128 * 4);
    float* sb = reinterpret_cast<float*>(own + kPatchBytes);
    uint32_t acc = 0;
    for (int t = pair; t < a.tiles; t += pairs, ++acc) {
      const uint32_t ab = acc & 1;
      int m0, n0;
      tile_origin(a, t, m0, n0);
      m0 += (int)rank * 128 + quad * 32;                  // this warp's rows and columns
      n0 += half * 128;
      const float sa = a.c.scale_a && m0 + lane < a.c.m ? __ldg(a.c.scale_a + m0 + lane) : 1.f;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int n = n0 + k * 32 + lane;
        sb[k * 32 + lane] = a.c.scale_b && n < a.c.n ? __ldg(a.c.scale_b + n) : 1.f;
      }
      __syncwarp();
      const bool got = mbar_wait(&tfull[ab], (acc >> 1) & 1, abort_flag, status);
      if (!__all_sync(0xffffffffu, got)) break;
      tcgen05_after_sync();
      const int rows = min(32, a.c.m - m0);
      if (a.c.out_fp32) store_tile<INT8, float>(a, trow + ab * kTile, sa, sb, own, m0, n0, rows);
      else store_tile<INT8, __nv_bfloat16>(a, trow + ab * kTile, sa, sb, own, m0, n0, rows);
      tcgen05_before_sync();
      __syncwarp();
      if (lane == 0) arrive_cluster(lead_tempty + 8u * ab);
    }
  }
  // Neither CTA leaves while its partner can still touch its shared or tensor memory.
  tcgen05_before_sync();
  __syncwarp();
  __syncthreads();
  cluster_barrier();
  if (warp == 1) {
    tcgen05_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

template <bool INT8, bool P_MN, bool Q_MN>
int launch_pairs(const CUtensorMap& mp, const CUtensorMap& mq, const PairArgs& a, cudaStream_t stream) {
  static PerDeviceOnce once;
  static int resident[64];
  int dev;
  if (once.need(&dev)) {
    if (dev < 0) return PRM_ERR_CUDA;
    const cudaError_t e = cudaFuncSetAttribute(matmul_q8_pair_kernel<INT8, P_MN, Q_MN>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
    if (e != cudaSuccess) return q8_code(e);
    const int n = q8_resident_clusters(matmul_q8_pair_kernel<INT8, P_MN, Q_MN>, kThreads, kSmemBytes, 2);
    if (n < 1) return PRM_ERR_CUDA;
    resident[dev] = n;
    once.mark(dev);
  }
  return q8_code(launch_after(matmul_q8_pair_kernel<INT8, P_MN, Q_MN>, 2u * (unsigned)std::min(a.tiles, resident[dev]),
                              kThreads, kSmemBytes, stream, 2, mp, mq, a));
}

}  // namespace

double matmul_q8_pairs_cycles(const MatmulProblem& p) {
  const double tiles = (double)((p.c.m + kTile - 1) / kTile) * ((p.c.n + kTile - 1) / kTile);
  if (tiles >= (1 << 30) || (p.int8 && p.c.kblocks > kMaxBlocksInt8)) return 1e30;
  // 512 cycles of matrix instructions per k-block of a tile; the epilogue of the last tile alone
  const double waves = std::ceil(tiles / 74);
  return std::max(waves * (p.c.kblocks * 520.0 + 1600), matmul_q8_memory_cycles(p)) + 4500;
}

int matmul_q8_pairs(const MatmulProblem& p) {
  PairArgs g = {};
  g.c = p.c;
  g.m_tiles = (p.c.m + kTile - 1) / kTile;
  g.n_tiles = (p.c.n + kTile - 1) / kTile;
  g.tiles = g.m_tiles * g.n_tiles;
  // As many m-tiles as keep their rows of a within 32 MB of the L2, at least 8 (a quarter of a wave).
  // With all m-tiles in one band 8192 x 16384 x 4096, whose a alone is larger than the L2, reads a
  // again for every wave.
  const int64_t fit = ((int64_t)32 << 20) / ((int64_t)kTile * p.c.kblocks * kBlockK);
  g.band = (int)std::min<int64_t>(g.m_tiles, std::max<int64_t>(8, fit));
  CUtensorMap mp, mq;
  if (!q8_make_map(&mp, p.a, p.a_rows, p.a_cols, p.ld_a, 128) ||
      !q8_make_map(&mq, p.b, p.b_rows, p.b_cols, p.ld_b, 128))
    return PRM_ERR_CUDA;
#define PRM_Q8_LAUNCH(I8, PM, QM) \
  if (p.int8 == I8 && p.a_t == PM && !p.b_t == QM) return launch_pairs<I8, PM, QM>(mp, mq, g, p.stream)
  PRM_Q8_LAUNCH(true, true, false);
  PRM_Q8_LAUNCH(true, false, false);
  PRM_Q8_LAUNCH(true, true, true);
  PRM_Q8_LAUNCH(true, false, true);
  PRM_Q8_LAUNCH(false, true, false);
  PRM_Q8_LAUNCH(false, false, false);
  PRM_Q8_LAUNCH(false, true, true);
  PRM_Q8_LAUNCH(false, false, true);
#undef PRM_Q8_LAUNCH
  return PRM_ERR_ARG;
}

}  // namespace prm
