// Product of 8-bit matrices with a scale per row of the left and per column of the right operand:
//
//   out[m, n] = scale_a[m] * scale_b[n] * sum_k a[m, k] * b[k, n]
//
// int8 codes are summed exactly in 32-bit integers, e4m3 codes in fp32.  Either operand may be
// stored either way round: a as rows of k or rows of m, b as rows of n or rows of k.  A layer's
// three products are then y = x8 W8, grad_x = g8 W8^T and grad_W = x8^T g8 on matrices as they lie.
//
// One CTA computes a tile of 128 columns n (the matrix instruction's M, so that a tensor-memory
// lane is an output column and a warp stores 32 neighbouring columns) by up to 256 rows m (its N):
// one token costs the instruction no more columns than it has to.  The k loop of a tile may be
// split over the CTAs of a cluster, which then add their parts through distributed shared memory:
// with few tiles this is what puts every SM on the weight's bytes.
//
//   warp 0      TMA producer: boxes of 128 bytes x 128 rows, 128-byte swizzle, no multicast
//   warp 1      tcgen05.mma issuer, owner of the tensor memory
//   warps 2..5  epilogue
//
// Every barrier wait is bounded; one that runs out sets the status word that prm_q8_status reads,
// the CTA drains its copies and leaves.
#include "q8_matmul.cuh"

namespace prm {
namespace {

__device__ int g_q8_status;

constexpr int kTileN = 128;            // output columns per CTA (lanes of the accumulator)
constexpr int kMaxStages = 10;
constexpr int kThreads = 192;
constexpr uint32_t kBytesP = kTileN * kBlockK;
constexpr int kMaxSplit = 8;           // portable cluster size

struct SplitArgs {
  MatmulArgs c;
  int tile_m;             // rows m per tile: 16, 32, 64, 128 or 256
  int n_tiles;
  int split;              // CTAs per tile (cluster size)
  int stages;
  uint32_t stage_bytes;
};

// Dynamic shared memory: stages (P tile, Q tile), reused for the split's partial sums.
template <bool INT8, bool P_MN, bool Q_MN>
__global__ void __launch_bounds__(kThreads, 1)
matmul_q8_kernel(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q,
                 const SplitArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  volatile int* abort_flag = &abort_word;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = a.split > 1 ? (int)cluster_ctarank() : 0;
  const int tile = blockIdx.x / a.split;
  const int n0 = (tile % a.n_tiles) * kTileN, m0 = (tile / a.n_tiles) * a.tile_m;
  const int kb0 = (int)((int64_t)a.c.kblocks * rank / a.split), kb1 = (int)((int64_t)a.c.kblocks * (rank + 1) / a.split);
  const uint32_t tmem_cols = a.tile_m < 32 ? 32u : (uint32_t)a.tile_m;

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(&done, 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)),
                 "r"(tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      int it = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        const int s = it % a.stages;
        if (!mbar_wait(&empty[s], ((it / a.stages) & 1) ^ 1, abort_flag, a.c.status)) break;
        uint8_t* sp = smem + (size_t)s * a.stage_bytes;
        uint8_t* sq = sp + kBytesP;
        mbar_expect_tx(&full[s], a.stage_bytes);
        const int k0 = kb * kBlockK;
        if (P_MN) tma_load_2d(sp, &map_p, &full[s], n0, k0);
        else tma_load_2d(sp, &map_p, &full[s], k0, n0);
        if (Q_MN) {
          tma_load_2d(sq, &map_q, &full[s], m0, k0);
          if (a.tile_m > 128) tma_load_2d(sq + 128 * kBlockK, &map_q, &full[s], m0 + 128, k0);
        } else {
          tma_load_2d(sq, &map_q, &full[s], k0, m0);
        }
      }
      if (*abort_flag) {                 // copies in flight must land before the CTA leaves
        for (int j = it > a.stages ? it - a.stages : 0; j < it; ++j) {
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(&full[j % a.stages], (j / a.stages) & 1) && global_ns() - t0 < 1000000ull) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_8bit(INT8, kTileN, a.tile_m, P_MN, Q_MN);
      constexpr uint32_t kStepP = P_MN ? 256 : 2, kStepQ = Q_MN ? 256 : 2;    // 32 k, in units of 16 bytes
      bool ok = true;
      int it = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        const int s = it % a.stages;
        if (!mbar_wait(&full[s], (it / a.stages) & 1, abort_flag, a.c.status)) { ok = false; break; }
        tcgen05_after_sync();
        const uint32_t sp = smem_u32(smem + (size_t)s * a.stage_bytes), sq = sp + kBytesP;
        const uint64_t dp = P_MN ? desc_mn_major(sp, 128 * kBlockK) : desc_k_major(sp);
        const uint64_t dq = Q_MN ? desc_mn_major(sq, 128 * kBlockK) : desc_k_major(sq);
#pragma unroll
        for (int j = 0; j < kBlockK / 32; ++j)
          umma_8bit_1cta<INT8>(tmem, dp + kStepP * j, dq + kStepQ * j, idesc, (it | j) != 0);
        umma_commit_1cta(&empty[s]);
      }
      if (ok) umma_commit_1cta(&done);
    }
  }
  bool ok = true;
  if (warp >= 2) {
    ok = mbar_wait(&done, 0, abort_flag, a.c.status);
    ok = __all_sync(0xffffffffu, ok);
    tcgen05_after_sync();
  }
  const int quad = warp & 3;
  const int col = quad * 32 + lane;            // this thread's output column in the tile
  const int n = n0 + col;
  const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
  const int m_here = min(a.tile_m, a.c.m - m0);
  const float sb = warp >= 2 && a.c.scale_b && n < a.c.n ? __ldg(a.c.scale_b + n) : 1.f;
  auto put = [&](int t, float v, float sa) {   // row t of this tile
    const int64_t at = (int64_t)(m0 + t) * a.c.ld_out + n;
    v = v * sa * sb;
    if (a.c.out_fp32) reinterpret_cast<float*>(a.c.out)[at] = v;
    else reinterpret_cast<__nv_bfloat16*>(a.c.out)[at] = __float2bfloat16_rn(v);
  };
  // The scale of row t, one per lane and handed round by shuffles: a load per row would serialise
  // on its latency.
  auto row_scale = [&](int t) {
    return a.c.scale_a && t < m_here ? __ldg(a.c.scale_a + m0 + t) : 1.f;
  };
  if (a.split == 1) {
    if (warp >= 2 && ok) {
      for (int t0 = 0; t0 < m_here; t0 += 16) {
        uint32_t r[16];
        tmem_ld16(trow + t0, r);
        const float sa = row_scale(t0 + (lane & 15));
        tmem_wait_ld();
        const int64_t at = (int64_t)(m0 + t0) * a.c.ld_out + n;
        if (a.c.out_fp32)
          store_column<INT8, 16>(reinterpret_cast<float*>(a.c.out) + at, a.c.ld_out, r, sa, sb, m_here - t0, n < a.c.n);
        else
          store_column<INT8, 16>(reinterpret_cast<__nv_bfloat16*>(a.c.out) + at, a.c.ld_out, r, sa, sb, m_here - t0,
                                 n < a.c.n);
      }
    }
  } else {
    uint32_t* part = reinterpret_cast<uint32_t*>(smem);       // [tile_m][128], all copies have been consumed
    if (warp >= 2 && ok) {
      for (int t0 = 0; t0 < m_here; t0 += 16) {
        uint32_t r[16];
        tmem_ld16(trow + t0, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) part[(t0 + j) * kTileN + col] = r[j];
      }
    }
    __syncwarp();
    cluster_barrier();
    if (warp >= 2 && ok) {
      // Rows t = rank, rank + split, ...: four at a time, so that their parts are fetched together.
      const uint32_t base = smem_u32(part) + (uint32_t)col * 4;
      for (int t0 = rank; t0 < m_here; t0 += 4 * a.split) {
        const float sa = row_scale(t0 + (lane & 3) * a.split);
        long long isum[4] = {0, 0, 0, 0};
        float fsum[4] = {0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < a.split; ++q) {
          const uint32_t at = cluster_map(base, q);
          uint32_t v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = t0 + j * a.split;
            v[j] = t < m_here ? ld_cluster_u32(at + (uint32_t)t * kTileN * 4) : 0u;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (INT8) isum[j] += (int)v[j];
            else fsum[j] += __uint_as_float(v[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s = __shfl_sync(0xffffffffu, sa, j);
          const int t = t0 + j * a.split;
          if (n < a.c.n && t < m_here) put(t, INT8 ? (float)isum[j] : fsum[j], s);
        }
      }
    }
    __syncwarp();
    cluster_barrier();                   // nobody leaves while its part is being read
  }
  tcgen05_before_sync();
  __syncwarp();
  __syncthreads();
  if (warp == 1) {
    tcgen05_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
  }
}

constexpr size_t kSmemBudget = 200 * 1024;

template <bool INT8, bool P_MN, bool Q_MN>
int launch_matmul(const CUtensorMap& mp, const CUtensorMap& mq, const SplitArgs& a, int ctas, size_t smem,
                  cudaStream_t stream) {
  static PerDeviceOnce once;
  int dev;
  if (once.need(&dev)) {
    if (cudaFuncSetAttribute(matmul_q8_kernel<INT8, P_MN, Q_MN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)(kSmemBudget + 1024)) != cudaSuccess)
      return PRM_ERR_CUDA;
    once.mark(dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)a.split;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, matmul_q8_kernel<INT8, P_MN, Q_MN>, mp, mq, a) == cudaSuccess ? PRM_OK
                                                                                              : PRM_ERR_CUDA;
}

int matmul_split(const MatmulProblem& p) {
  const int64_t m = p.c.m, n = p.c.n;
  SplitArgs g = {};
  g.c = p.c;
  g.tile_m = 16;
  while (g.tile_m < 256 && g.tile_m < m) g.tile_m *= 2;
  g.n_tiles = (int)((n + kTileN - 1) / kTileN);
  const int64_t tiles = (int64_t)g.n_tiles * ((m + g.tile_m - 1) / g.tile_m);
  // Split k while every SM would otherwise not get a tile, but leave each CTA four k-blocks.
  int split = 1;
  while (split < kMaxSplit && tiles * (split + 1) <= 148 && g.c.kblocks >= 4 * (split + 1)) ++split;
  if (p.int8) {
    const int need = (g.c.kblocks + kMaxBlocksInt8 - 1) / kMaxBlocksInt8;
    if (need > kMaxSplit) return PRM_ERR_SHAPE;
    split = std::max(split, need);
  }
  g.split = split;
  if (tiles * split > 0x7fffffffLL) return PRM_ERR_SHAPE;
  const uint32_t q_bytes = (p.a_t ? (uint32_t)std::max(g.tile_m, 128) : (uint32_t)g.tile_m) * kBlockK;
  g.stage_bytes = kBytesP + q_bytes;
  const int blocks_each = (g.c.kblocks + split - 1) / split;
  g.stages = std::max(1, std::min<int>({kMaxStages, blocks_each, (int)(kSmemBudget / g.stage_bytes)}));
  size_t smem = (size_t)g.stages * g.stage_bytes;
  if (split > 1) smem = std::max(smem, (size_t)g.tile_m * kTileN * 4);
  smem += 1024;
  CUtensorMap mp, mq;
  if (!q8_make_map(&mp, p.b, p.b_rows, p.b_cols, p.ld_b, 128) ||
      !q8_make_map(&mq, p.a, p.a_rows, p.a_cols, p.ld_a, p.a_t ? 128 : g.tile_m))
    return PRM_ERR_CUDA;
  const int ctas = (int)(tiles * split);
#define PRM_Q8_LAUNCH(I8, PM, QM) \
  if (p.int8 == I8 && !p.b_t == PM && p.a_t == QM) return launch_matmul<I8, PM, QM>(mp, mq, g, ctas, smem, p.stream)
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

}  // namespace

// The status word's address on the current device.
int* q8_status_word() {
  static int* at[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  if (!at[dev]) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_q8_status) != cudaSuccess) return nullptr;
    at[dev] = (int*)p;
  }
  return at[dev];
}

}  // namespace prm

using namespace prm;

extern "C" int prm_matmul_q8(const void* a, int64_t ld_a, int a_transposed, const float* scale_a, const void* b,
                             int64_t ld_b, int b_transposed, const float* scale_b, int64_t m, int64_t k, int64_t n,
                             int format, void* out, int64_t ld_out, int out_fp32, void* cuda_stream) {
  if (!q8_format_ok(format)) return PRM_ERR_ARG;
  const int64_t most = 0x7fffffffLL - 1024;
  if (m < 0 || n < 0 || k < 0 || m > most || n > most || k > most) return PRM_ERR_SHAPE;
  if (m == 0 || n == 0) return PRM_OK;
  if (!out) return PRM_ERR_ARG;
  const int es = out_fp32 ? 4 : 2;
  if (ld_out < n || ld_out > ((int64_t)1 << 40)) return PRM_ERR_SHAPE;
  if ((uintptr_t)out % es != 0 || ((uintptr_t)scale_a | (uintptr_t)scale_b) % 4 != 0) return PRM_ERR_ALIGN;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (k == 0)                             // an empty sum
    return cudaMemset2DAsync(out, (size_t)ld_out * es, 0, (size_t)n * es, (size_t)m, stream) == cudaSuccess
               ? PRM_OK
               : PRM_ERR_CUDA;
  if (!a || !b) return PRM_ERR_ARG;
  const int64_t a_rows = a_transposed ? k : m, a_cols = a_transposed ? m : k;
  const int64_t b_rows = b_transposed ? n : k, b_cols = b_transposed ? k : n;
  if (ld_a < a_cols || ld_b < b_cols || ld_a >= ((int64_t)1 << 39) || ld_b >= ((int64_t)1 << 39)) return PRM_ERR_SHAPE;
  if (!aligned16(a) || !aligned16(b) || ld_a % 16 != 0 || ld_b % 16 != 0) return PRM_ERR_ALIGN;

  const bool p_mn = !b_transposed, q_mn = a_transposed != 0;
  MatmulProblem p = {};
  p.c = {scale_a, scale_b, out, q8_status_word(), ld_out, (int)m, (int)n, (int)((k + kBlockK - 1) / kBlockK), out_fp32};
  p.a = a;
  p.b = b;
  p.ld_a = ld_a;
  p.ld_b = ld_b;
  p.a_rows = a_rows;
  p.a_cols = a_cols;
  p.b_rows = b_rows;
  p.b_cols = b_cols;
  p.a_t = q_mn;
  p.b_t = !p_mn;
  p.int8 = format == PRM_Q8_INT8;
  p.stream = stream;
  if (!p.c.status) return PRM_ERR_CUDA;
  if (matmul_q8_wants_pairs(p)) return matmul_q8_pairs(p);
  return matmul_split(p);
}

extern "C" int prm_q8_status(void) {
  int v = 0;
  const int zero = 0;
  if (cudaDeviceSynchronize() != cudaSuccess) return PRM_ERR_CUDA;
  if (cudaMemcpyFromSymbol(&v, g_q8_status, sizeof(int)) != cudaSuccess) return PRM_ERR_CUDA;
  if (v == 0) return PRM_OK;
  if (cudaMemcpyToSymbol(g_q8_status, &zero, sizeof(int)) != cudaSuccess) return PRM_ERR_CUDA;
  return PRM_ERR_DEVICE_TIMEOUT;
}
