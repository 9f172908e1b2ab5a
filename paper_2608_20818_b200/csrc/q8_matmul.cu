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
//   warps 2..9  epilogue: two warps per lane quadrant, every other set of 16 rows m each
//
// Every barrier wait is bounded; one that runs out sets the status word that prm_q8_status reads,
// the CTA drains its copies and leaves.
#include <type_traits>

#include "q8_matmul.cuh"
#include "q8_plan.h"

namespace prm {
namespace {

__device__ int g_q8_status;

constexpr int kTileN = 128;            // output columns per CTA (lanes of the accumulator)
constexpr int kMaxStages = 10;
constexpr int kThreads = 320;
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

  auto load = [&](int kb, int s) {               // k-block kb into stage s
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
  };
  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(&done, 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    grid_wait();
    // the first copies need nobody else
    for (int it = 0; it < a.stages && kb0 + it < kb1; ++it) load(kb0 + it, it);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)),
                 "r"(tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcgen05_before_sync();
  __syncwarp();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = tmem_slot;
  grid_wait();
  grid_trigger();                              // not before the tensor memory is this kernel's

  if (warp == 0) {
    if (lane == 0) {
      int it = min(a.stages, kb1 - kb0);
      for (; kb0 + it < kb1; ++it) {
        const int s = it % a.stages;
        if (!mbar_wait(&empty[s], ((it / a.stages) & 1) ^ 1, abort_flag, a.c.status)) break;
        load(kb0 + it, s);
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
  const int quad = warp & 3, half = (warp - 2) >> 2;
  const int col = quad * 32 + lane;            // this thread's output column in the tile
  const int n = n0 + col;
  const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
  const int m_here = min(a.tile_m, a.c.m - m0);
  const float sb = warp >= 2 && a.c.scale_b && n < a.c.n ? __ldg(a.c.scale_b + n) : 1.f;
  // The scales of 16 rows from t on, one per lane and handed round by shuffles: a load per row would
  // serialise on its latency.
  auto row_scales = [&](int t) {
    t += lane & 15;
    return a.c.scale_a && t < m_here ? __ldg(a.c.scale_a + m0 + t) : 1.f;
  };
  // Rows t .. t + rows - 1 of the tile; `ints`: integer sums.
  auto store = [&](auto ints, int t, const uint32_t (&r)[16], float sa, int rows) {
    const int64_t at = (int64_t)(m0 + t) * a.c.ld_out + n;
    float* out_f = reinterpret_cast<float*>(a.c.out) + at;
    __nv_bfloat16* out_h = reinterpret_cast<__nv_bfloat16*>(a.c.out) + at;
    if (a.c.out_fp32) store_column<decltype(ints)::value, 16>(out_f, a.c.ld_out, r, sa, sb, rows, n < a.c.n);
    else store_column<decltype(ints)::value, 16>(out_h, a.c.ld_out, r, sa, sb, rows, n < a.c.n);
  };
  using Sums = std::integral_constant<bool, INT8>;
  if (a.split == 1) {
    if (warp >= 2 && ok) {
      for (int t = half * 16; t < m_here; t += 32) {
        uint32_t r[16];
        tmem_ld16(trow + t, r);
        const float sa = row_scales(t);
        tmem_wait_ld();
        store(Sums(), t, r, sa, m_here - t);
      }
    }
  } else {
    // CTA q of the cluster finishes rows q * own .. of the tile: every CTA writes its part of them into
    // q's shared memory (stores, so that nobody waits for a far load), then q adds what lies at home.
    // The stages may be overwritten once all CTAs' matrix instructions are done.
    const int own = ((m_here + a.split - 1) / a.split + 15) / 16 * 16;
    const uint32_t part = smem_u32(smem);        // [split][own][128]
    __syncwarp();
    cluster_barrier();
    if (warp >= 2 && ok) {
      for (int t = half * 16; t < m_here; t += 32) {
        uint32_t r[16];
        tmem_ld16(trow + t, r);
        const int q = t / own;                   // 16 rows have one owner
        const uint32_t at = cluster_map(part + (uint32_t)((rank * own + t - q * own) * kTileN + col) * 4, q);
        tmem_wait_ld();
        if (m_here - t >= 16) {
#pragma unroll
          for (int j = 0; j < 16; ++j) st_cluster_u32(at + j * kTileN * 4, r[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (t + j < m_here) st_cluster_u32(at + j * kTileN * 4, r[j]);
        }
      }
    }
    __syncwarp();
    cluster_barrier();
    if (warp >= 2 && ok) {
      const uint32_t* home = reinterpret_cast<const uint32_t*>(smem) + col;
      const int mine = min(own, m_here - rank * own);
      for (int t = half * 16; t < mine; t += 32) {
        const float sa = row_scales(rank * own + t);
        uint32_t sum[16];
        if (INT8) {
          // the parts' sum may leave 32 bits only where k is too long for one of them
          if (a.c.kblocks <= kMaxBlocksInt8) {
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[j] = 0;
            for (int q = 0; q < a.split; ++q)
#pragma unroll
              for (int j = 0; j < 16; ++j) sum[j] += home[(q * own + t + j) * kTileN];
            store(Sums(), rank * own + t, sum, sa, mine - t);
            continue;
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            long long v = 0;
            for (int q = 0; q < a.split; ++q) v += (int)home[(q * own + t + j) * kTileN];
            sum[j] = __float_as_uint((float)v);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[j] = 0;
          for (int q = 0; q < a.split; ++q)
#pragma unroll
            for (int j = 0; j < 16; ++j)
              sum[j] = __float_as_uint(__uint_as_float(sum[j]) + __uint_as_float(home[(q * own + t + j) * kTileN]));
        }
        store(std::false_type(), rank * own + t, sum, sa, mine - t);
      }
    }
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
    const cudaError_t e = cudaFuncSetAttribute(matmul_q8_kernel<INT8, P_MN, Q_MN>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kSmemBudget + 1024));
    if (e != cudaSuccess) return q8_code(e);
    once.mark(dev);
  }
  return q8_code(launch_after(matmul_q8_kernel<INT8, P_MN, Q_MN>, (unsigned)ctas, kThreads, smem, stream,
                              (unsigned)a.split, mp, mq, a));
}

// CTAs in clusters of `split` that are resident at once (1 per SM; how many clusters fit depends on how
// many SMs the GPCs have).
int resident_ctas(int split) {
  static int at[64][kMaxSplit + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (at[dev][split] == 0) {
    if (cudaFuncSetAttribute(matmul_q8_kernel<true, true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)(kSmemBudget + 1024)) != cudaSuccess)
      return 0;
    at[dev][split] =
        split * q8_resident_clusters(matmul_q8_kernel<true, true, false>, kThreads, kSmemBudget + 1024, (unsigned)split);
  }
  return at[dev][split];
}

struct Plan {
  int tile_m = 0, split = 0;
  double cycles = 1e30;
};

// Which tile height and how many CTAs to a tile: the cheapest of all by an estimate of SM cycles, with
// the rates measured on a B200: 2 tile_m cycles of matrix instructions per k-block, 60 bytes per cycle
// and SM from L2, 24 cycles per row of the epilogue.
Plan plan_split(const MatmulProblem& p) {
  Plan best;
  const int need = p.int8 ? (p.c.kblocks + kMaxBlocksInt8 - 1) / kMaxBlocksInt8 : 1;
  const double memory = matmul_q8_memory_cycles(p);
  const int64_t n_tiles = (p.c.n + kTileN - 1) / kTileN;
  for (int tile_m = 16; tile_m <= 256; tile_m *= 2) {
    const int64_t tiles = n_tiles * ((p.c.m + tile_m - 1) / tile_m);
    for (int split = need; split <= kMaxSplit && (split == need || split * 2 <= p.c.kblocks); ++split) {
      const int slots = resident_ctas(split);
      if (slots < 1) continue;
      const double waves = std::ceil((double)tiles * split / slots);
      if (waves > 1 && split > need) break;
      const int blocks = (p.c.kblocks + split - 1) / split;
      const double block = std::max(2.0 * tile_m, (128.0 + tile_m) * kBlockK / 60);
      const double tail = split > 1 ? 1200 + 12.0 * tile_m + 24.0 * tile_m / split : 24.0 * tile_m;
      const double cycles = std::max(waves * blocks * block, memory) + waves * tail + (waves - 1) * 4000;
      if (cycles < best.cycles) best = {tile_m, split, cycles};
    }
    if (tile_m >= p.c.m) break;
  }
  return best;
}

int matmul_split(const MatmulProblem& p, const Plan& plan) {
  const int64_t m = p.c.m, n = p.c.n;
  SplitArgs g = {};
  g.c = p.c;
  g.tile_m = plan.tile_m;
  g.split = plan.split;
  g.n_tiles = (int)((n + kTileN - 1) / kTileN);
  const int64_t tiles = (int64_t)g.n_tiles * ((m + g.tile_m - 1) / g.tile_m);
  const int split = g.split;
  if (tiles * split > 0x7fffffffLL) return PRM_ERR_SHAPE;
  const uint32_t q_bytes = (p.a_t ? (uint32_t)std::max(g.tile_m, 128) : (uint32_t)g.tile_m) * kBlockK;
  g.stage_bytes = kBytesP + q_bytes;
  const int blocks_each = (g.c.kblocks + split - 1) / split;
  g.stages = std::max(1, std::min<int>({kMaxStages, blocks_each, (int)(kSmemBudget / g.stage_bytes)}));
  size_t smem = (size_t)g.stages * g.stage_bytes;
  if (split > 1) smem = std::max(smem, (size_t)(g.tile_m + 16 * split) * kTileN * 4);
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

int q8_sms() {
  static int at[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  int sms = 0;
  if (!at[dev] && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
    at[dev] = std::min(sms, kRingBlocks);
  return at[dev];
}

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
    return q8_code(cudaMemset2DAsync(out, (size_t)ld_out * es, 0, (size_t)n * es, (size_t)m, stream));
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
  if (p.int8 && p.c.kblocks > kMaxSplit * kMaxBlocksInt8) return PRM_ERR_SHAPE;
  if (!p.c.status) return PRM_ERR_CUDA;
  const Plan plan = plan_split(p);
  if (matmul_q8_pairs_cycles(p) < plan.cycles) return matmul_q8_pairs(p);
  return plan.tile_m > 0 ? matmul_split(p, plan) : PRM_ERR_CUDA;
}

extern "C" int prm_q8_status(void) {
  int v = 0;
  const int zero = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&v, g_q8_status, sizeof(int));
  if (e == cudaSuccess && v != 0) e = cudaMemcpyToSymbol(g_q8_status, &zero, sizeof(int));
  return e != cudaSuccess ? q8_code(e) : v != 0 ? PRM_ERR_DEVICE_TIMEOUT : PRM_OK;
}
