// Softmax cross entropy of a linear head, without keeping its logits:
//
//   l = x W;   lse_i = log sum_v exp l_iv;   loss_i = lse_i - l_i,label
//   G_iv = gl_i (exp(l_iv - lse_i) - [v = label_i]);   grad_x = G W^T;   grad_W = x^T G
//
// Bound by the tensor pipe (2 n d V flop forward, 6 n d V backward, two of them for the logits again), with
// few rows by W's bytes.  The logits live in tensor memory only.  Forward, the epilogue of a tile leaves two numbers per
// row and 128 columns, the largest logit and the sum of exponentials relative to it; a second kernel joins them.
// Backward, G exists for a piece of the vocabulary at a time, as an operand of the two products that follow.
//
// G is rounded to bf16, the type of the operands that it is multiplied with (relative 2^-8 at most, of each entry by
// itself); the factor of the rows' gradients is kept out of it: G is made of gl_i / c with c = max |gl|, which is
// exactly 1 for a mean or a sum, and the products' fp32 sums are multiplied by c.  All else is fp32, rounded once.
//
// All products run in one kernel on pairs of CTAs (tcgen05.mma.cta_group::2), 256 x 256 tiles:
//   warp 0      TMA producer: per stage 128 k of both operands (64 KB), 128-byte swizzle, no multicast; the
//               copies of both CTAs count on the leader's barrier.  Three stages
//   warp 1      tcgen05.mma issuer (one lane of the leader); owns its CTA's tensor memory
//   warps 2..9  epilogue: two warps per lane quadrant, half of the 256 columns each; a thread has a row
// Two accumulators of 256 columns let the epilogue of a tile run under the next tile's main loop.
// Measured, one after another: 8192 x 4096 x 131072 6.4 ms, 1370 TFLOP/s, its gradient with 65536 columns 10.4 ms, 1265 TFLOP/s
// (cuBLAS sustains 1374 under the same power cap); 2048 x 1024 x 32768 103 us and 319 us; one token 4096 x 32768 52 us, 5.1 TB/s.
// Every barrier wait is bounded; one that runs out sets the status word, the pair drains and leaves.
#include "q8_matmul.cuh"
#include "train_plan.h"

namespace prm {
namespace {

constexpr int kTile = kHeadTile;                 // tile edge, both ways
constexpr int kHeadK = 64;                       // one 128-byte swizzled row of k
constexpr int kSub = 2;                          // k-blocks per stage
constexpr int kStages = 3;
static_assert(kHeadStage == kSub * kHeadK, "the plan's stage");
constexpr int kEpiWarps = 8;
constexpr int kThreads = 32 * (2 + kEpiWarps);
constexpr uint32_t kBoxBytes = 128 * 128;        // 128 rows of one k-block
constexpr uint32_t kStageBytes = 2 * kSub * kBoxBytes;
constexpr uint32_t kPatchBytes = 32 * 64;        // a warp's 32 rows of 64 bytes on their way out
constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + kEpiWarps * kPatchBytes;
constexpr int kMaxStages = 6;
constexpr int kFewRows = 64;                     // rows that kFew takes (100 x 4096 x 32768: 4 us more than the other form)
// Long sums are taken out of tensor memory every so often and added in registers: the accumulator cuts off what falls below its
// last bit at each of its steps (16 k).  The logits' every 1024 k, in both directions, so that the gradient's are those that
// lse was made of: over 4096 k a logit of the size 1 would be off by 1e-5 (it costs the gradient of 100 x 4096 x 32768 3 %).
// Those of the products of G, which are rounded to bf16 in the end, every 8192 k where there are more than 32768 (up to there
// what is cut off is 2e-4 of a sum of one sign, a twentieth of its rounding; over 2^20 rows grad_W would be 6e-3 short).
constexpr int kLogitChunk = 8, kStoreChunk = 64; // stages
constexpr int kStoreLongest = 256;
constexpr float kLog2e = 1.4426950408889634f;

// kStats: x (rows) times W (columns).  kFew: the same for few rows, the other way round (the rows are the instruction's N, so
// that it costs them no more than it has to, and W's bytes have most of shared memory).
// kGradLong, kStoreLong: tiles of several chunks (in one kernel with the others their registers cost 8192 x 64 x 32768 550 us
// instead of 470).
enum Epi { kStats, kFew, kGrad, kGradLong, kStore, kStoreLong };
__host__ __device__ constexpr bool is_grad(int epi) { return epi == kGrad || epi == kGradLong; }
__host__ __device__ constexpr bool is_store(int epi) { return epi == kStore || epi == kStoreLong; }
// Stages of a chunk: all of a tile's, where it is one.
__host__ __device__ constexpr int chunk_of(int epi) {
  return epi == kGrad || epi == kStore ? 1 << 30 : epi == kStoreLong ? kStoreChunk : kLogitChunk;
}

struct HeadArgs {
  int m, n, kblocks;               // of this product: rows, columns, ceil(k / 64)
  int p_mn, q_mn;                  // kStore: the operand's m (n) is contiguous, not its k
  int q_n0, q_k0;                  // where it starts in Q
  int m_tiles, n_tiles, tiles;     // tiles: of all splits of k
  int band;                        // m-tiles that are walked through together
  int split;                       // parts of k (kStore)
  int q_tile, stages;              // kFew: N of the instruction, stages that fit
  uint32_t stage_bytes;
  int* status;
  // kStats, kGrad
  const int64_t* labels;
  int64_t vocab;
  float2* part;                    // [2 n_tiles][m] (kFew: [ceil(vocab / 256) 8][n]): largest logit, sum of e^(logit - that)
  float* at_label;                 // of each row
  const float* lse;
  const float* grad_loss;
  __nv_bfloat16* g;
  int64_t ld_g;
  const __nv_bfloat16* x;          // kGrad: where x is to be copied to without the rows that have no part, else null
  __nv_bfloat16* clean;
  int64_t ld_x, ld_clean;
  int d;
  // kGrad, kStore
  const float* unit;               // c; null: 1
  float* unit_out;                 // kGrad: c is computed by every block, and left here (kUnitRows rows at most)
  void* out;
  int64_t ld_out, split_stride;
  int out_fp32, accumulate;        // accumulate: fp32 out += (16-byte aligned)
};

// A launch: one product, or (kStore) two that do not depend on one another.
struct HeadLaunch {
  CUtensorMap p[2], q[2];
  HeadArgs a[2];
  int extra;                       // see pair_tile
};

template <int EPI>
__device__ __forceinline__ bool next_tile(const HeadLaunch& l, int pair, int pairs, int i, int& which, int& tile) {
  if constexpr (is_store(EPI)) return pair_tile(l.a[0].tiles, l.a[1].tiles, l.extra, pair, pairs, i, which, tile);
  which = 0;
  tile = pair + i * pairs;
  return tile < l.a[0].tiles;
}

__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// e^(v - top), of two logits.  The difference comes first: it is exact next to top and gives top itself a share of exactly 1, so
// that no sum is below 1 and a row that is predicted with certainty has the loss 0.
__device__ __forceinline__ float2 share2(float2 v, float2 minus_top) {
  v = mul2(add2(v, minus_top), make_float2(kLog2e, kLog2e));
  return make_float2(ex2(v.x), ex2(v.y));
}

// Order of the tiles: bands of `band` m-tiles, in a band n by n, m-tiles fastest; the splits of k one after
// the other.  Pairs that run at the same time then share the band's rows of P and a few columns' worth of Q.
__device__ __forceinline__ void tile_origin(const HeadArgs& a, int t, int& split, int& m0, int& n0) {
  const int each = a.m_tiles * a.n_tiles;
  split = t / each;
  t -= split * each;
  const int per = a.band * a.n_tiles, first = t / per * a.band, rest = t % per;
  const int height = min(a.band, a.m_tiles - first);
  m0 = (first + rest % height) * kTile;
  n0 = rest / height * kTile;
}
__device__ __forceinline__ void split_range(const HeadArgs& a, int split, int& s0, int& s1) {
  head_part((a.kblocks + kSub - 1) / kSub, a.split, split, s0, s1);
}

// The label of a row as a column of the 128 from n0 on, -1 if it is none of them.
__device__ __forceinline__ int label_column(const HeadArgs& a, int64_t label, int n0) {
  const int64_t c = label - a.q_n0 - n0;
  return label >= 0 && label < a.vocab && c >= 0 && c < 128 ? (int)c : -1;
}

// 128 columns of the lane's row: what they add to the softmax, and the label's logit.
__device__ __forceinline__ void stats_tile(const HeadArgs& a, float (&v)[128], int row, int n0, int column) {
  const int label = row < a.m ? label_column(a, a.labels[row], n0) : -1;
  const int wide = a.n - n0;
  if (wide < 128) {
#pragma unroll
    for (int j = 0; j < 128; ++j)
      if (j >= wide) v[j] = -INFINITY;
  }
  float t[4] = {v[0], v[1], v[2], v[3]}, s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 4; j < 128; ++j) t[j & 3] = fmaxf(t[j & 3], v[j]);
  const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
  const float off = top == -INFINITY ? 0.f : -top;
#pragma unroll
  for (int j = 0; j < 128; j += 2) {
    const float2 e = share2(make_float2(v[j], v[j + 1]), make_float2(off, off));
    s[j & 3] += e.x;
    s[(j + 1) & 3] += e.y;
  }
  if (__any_sync(0xffffffffu, label >= 0)) {
#pragma unroll
    for (int j = 0; j < 128; ++j)
      if (label == j) a.at_label[row] = v[j];
  }
  if (row < a.m)
    a.part[(int64_t)column * a.m + row] = make_float2(top, (s[0] + s[1]) + (s[2] + s[3]));
}

// kFew: 32 columns (lanes) of 16 rows from n0 on.  They pass through shared memory, so that a lane gets 16 columns of one row.
__device__ __forceinline__ void few_tile(const HeadArgs& a, const float* v, float* patch, int m0, int n0) {
  const int lane = threadIdx.x & 31, r = lane & 15, part = lane >> 4, row = n0 + r;
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 16; ++k) patch[k * 32 + (lane ^ k)] = m0 + lane < a.m ? v[k] : -INFINITY;
  __syncwarp();
  float t[16], top = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    t[j] = patch[r * 32 + ((part * 16 + j) ^ r)];
    top = fmaxf(top, t[j]);
  }
  top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
  const float off = top == -INFINITY ? 0.f : -top;
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    const float2 e = share2(make_float2(t[j], t[j + 1]), make_float2(off, off));
    s += e.x;
    s += e.y;
  }
  s += __shfl_xor_sync(0xffffffffu, s, 16);
  if (row < a.n && part == 0) {
    a.part[(int64_t)(m0 / 32) * a.n + row] = make_float2(top, s);
    const int64_t c = a.labels[row] - m0;
    if (c >= 0 && c < 32 && c + m0 < a.vocab) a.at_label[row] = patch[r * 32 + ((int)c ^ r)];
  }
}

// 16-byte chunk c of row r of a warp's patch, where neither writing rows nor reading them back meets a bank twice.
__device__ __forceinline__ uint4* patch_at(uint8_t* patch, int r, int c) {
  return reinterpret_cast<uint4*>(patch + (r >> 1) * 128 + (r & 1) * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

// c = max |gl| over the rows with a label, 1 if that is 0 or no number: THREADS threads' share.
template <int THREADS>
__device__ __forceinline__ float unit_share(const float* grad_loss, const int64_t* labels, int64_t vocab, int rows, int thread) {
  float top = 0.f;
#pragma unroll 4
  for (int i = thread; i < rows; i += THREADS) {
    const int64_t l = labels[i];
    const float v = grad_loss[i];
    if (l >= 0 && l < vocab) top = fmaxf(top, fabsf(v));
  }
  return group_top(top);
}
__device__ __forceinline__ float unit_of(float top) { return top > 0.f && top < INFINITY ? top : 1.f; }
constexpr int kUnitRows = 2048;                  // for more it has a launch of its own

// Rows first, first + rows_apart, ... of x, one by one, to `clean`: zeros for a row without a label or with the gradient 0.  grad_W's sums
// run over the rows; what such a row of x holds (padding, which may be no number) must not reach them, not even times 0.
__device__ __forceinline__ void copy_live_rows(const HeadArgs& a, int first, int rows_apart) {
  const int lane = threadIdx.x & 31, octs = (a.d + 7) / 8;
  for (int64_t row = first; row < a.m; row += rows_apart) {
    const int64_t l = a.labels[row];
    const bool live = l >= 0 && l < a.vocab && a.grad_loss[row] != 0.f;
    const __nv_bfloat16* x = a.x + row * a.ld_x;
    uint4* to = reinterpret_cast<uint4*>(a.clean + row * a.ld_clean);
#pragma unroll 4
    for (int o = lane; o < octs; o += 32) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (live && o * 8 + 8 <= a.d) {
        v = *reinterpret_cast<const uint4*>(x + o * 8);
      } else if (live) {                   // what lies behind the row may be no memory of x
        const uint16_t* e = reinterpret_cast<const uint16_t*>(x + o * 8);
        uint32_t h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) h[k] = o * 8 + k < a.d ? e[k] : 0;
        v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
      }
      to[o] = v;
    }
  }
}

// 128 columns of the lane's row of G.
__device__ __forceinline__ void grad_tile(const HeadArgs& a, uint32_t taddr, uint8_t* patch, int m0, int n0, int rows,
                                          float unit) {
  const int lane = threadIdx.x & 31, row = m0 + lane;
  float factor = 0.f, off = 0.f;
  int label = -1;
  if (row < a.m) {
    const int64_t l = a.labels[row];
    if (l >= 0 && l < a.vocab) {
      factor = __fdiv_rn(a.grad_loss[row], unit);
      off = -a.lse[row];
      label = label_column(a, l, n0);
    }
  }
  const bool all = __all_sync(0xffffffffu, factor != 0.f);
  __nv_bfloat16* out = a.g + (int64_t)m0 * a.ld_g + n0;
#pragma unroll 1
  for (int k = 0; k < 4; ++k) {
    if (n0 + k * 32 >= a.n) break;
    uint32_t r[32];
    tmem_ld32(taddr + k * 32, r);
    tmem_wait_ld();
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
      const float2 e = share2(make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), make_float2(off, off));
      v[j] = e.x;
      v[j + 1] = e.y;
    }
    if (__any_sync(0xffffffffu, label >= k * 32 && label < k * 32 + 32)) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] -= label == k * 32 + j ? 1.f : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] *= factor;
    if (!all) {                            // a row without a label has no part, whatever its logits
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = factor == 0.f ? 0.f : v[j];
    }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *patch_at(patch, lane, c) =
          make_uint4(pair_to_bf16(make_float2(v[c * 8], v[c * 8 + 1])), pair_to_bf16(make_float2(v[c * 8 + 2], v[c * 8 + 3])),
                     pair_to_bf16(make_float2(v[c * 8 + 4], v[c * 8 + 5])), pair_to_bf16(make_float2(v[c * 8 + 6], v[c * 8 + 7])));
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = i * 8 + (lane >> 2);
      const uint4 x = *patch_at(patch, at, lane & 3);
      if (at < rows) *reinterpret_cast<uint4*>(out + at * a.ld_g + k * 32 + (lane & 3) * 8) = x;   // rows are padded to 64
    }
  }
}

// 128 columns of the lane's row of a product.
template <typename OUT>
__device__ __forceinline__ void store_tile(const HeadArgs& a, uint32_t taddr, uint8_t* patch, int split, int m0, int n0,
                                           int rows, float unit) {
  constexpr int kCols = 64 / sizeof(OUT);                 // per piece
  const int lane = threadIdx.x & 31;
  OUT* out = reinterpret_cast<OUT*>(a.out) + split * a.split_stride + (int64_t)m0 * a.ld_out + n0;
  const bool vec = ((uintptr_t)out & 15) == 0 && (a.ld_out * (int64_t)sizeof(OUT)) % 16 == 0;
  const bool by4 = ((uintptr_t)out & 3) == 0 && a.ld_out % 2 == 0;
#pragma unroll 1
  for (int k = 0; k < 4; ++k) {
    if (n0 + k * 32 >= a.n) break;
    uint32_t r[32];
    tmem_ld32(taddr + k * 32, r);
    tmem_wait_ld();
#pragma unroll
    for (int piece = 0; piece < 32 / kCols; ++piece) {
      const int wide = min(kCols, a.n - (n0 + k * 32 + piece * kCols));
      if (wide <= 0) break;
      uint4 w[4];
      uint32_t* o = reinterpret_cast<uint32_t*>(w);
#pragma unroll
      for (int c = 0; c < kCols; c += 2) {
        const float2 u = mul2(make_float2(__uint_as_float(r[piece * kCols + c]), __uint_as_float(r[piece * kCols + c + 1])),
                              make_float2(unit, unit));
        if constexpr (sizeof(OUT) == 2) {
          o[c / 2] = pair_to_bf16(u);
        } else {
          o[c] = __float_as_uint(u.x);
          o[c + 1] = __float_as_uint(u.y);
        }
      }
      __syncwarp();                                       // the piece before has been read
#pragma unroll
      for (int c = 0; c < 4; ++c) *patch_at(patch, lane, c) = w[c];
      __syncwarp();
      OUT* to = out + k * 32 + piece * kCols;
      if (vec && wide == kCols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = i * 8 + (lane >> 2);
          uint4 x = *patch_at(patch, row, lane & 3);
          if (row < rows) {
            uint4* p = reinterpret_cast<uint4*>(to + row * a.ld_out + (lane & 3) * (16 / sizeof(OUT)));
            if constexpr (sizeof(OUT) == 4) {
              if (a.accumulate) {
                const float4 old = *reinterpret_cast<const float4*>(p);
                x = make_uint4(__float_as_uint(old.x + __uint_as_float(x.x)), __float_as_uint(old.y + __uint_as_float(x.y)),
                               __float_as_uint(old.z + __uint_as_float(x.z)), __float_as_uint(old.w + __uint_as_float(x.w)));
              }
            }
            *p = x;
          }
        }
      } else if (sizeof(OUT) == 2 && by4 && wide == kCols) {     // rows that start on 4 bytes: two columns per lane
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
          const int row = i * 2 + (lane >> 4), c = (lane & 15) * 4;
          if (row < rows)
            *reinterpret_cast<uint32_t*>(to + row * a.ld_out + c / 2) =
                *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(patch_at(patch, row, c >> 4)) + (c & 15));
        }
      } else {
#pragma unroll 4
        for (int row = 0; row < rows; ++row) {
          const int c = lane * (int)sizeof(OUT);
          if (lane < wide) {
            OUT v = *reinterpret_cast<const OUT*>(reinterpret_cast<const uint8_t*>(patch_at(patch, row, (c >> 4) & 3)) + (c & 15));
            if constexpr (sizeof(OUT) == 4) {
              if (a.accumulate) v += to[row * a.ld_out + lane];
            }
            to[row * a.ld_out + lane] = v;
          }
        }
      }
    }
  }
}

// A thread's 128 sums in tensor memory: added to v, and set.
__device__ __forceinline__ void add_sums(uint32_t taddr, float (&v)[128]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t r[32];
    tmem_ld32(taddr + k * 32, r);
    tmem_wait_ld();
#pragma unroll
    for (int j = 0; j < 32; ++j) v[k * 32 + j] += __uint_as_float(r[j]);
  }
}
__device__ __forceinline__ void put_sums(uint32_t taddr, const float (&v)[128]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t r[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(v[k * 32 + j]);
    tmem_st32(taddr + k * 32, r);
  }
  tmem_wait_st();
}

// P_MN, Q_MN: as HeadArgs has them (kStore goes by those).
template <int EPI, bool P_MN, bool Q_MN>
__global__ void __launch_bounds__(kThreads, 1) head_kernel(const __grid_constant__ HeadLaunch l) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  volatile int* abort_flag = &abort_word;
  int* status = l.a[0].status;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int stages = EPI == kFew ? l.a[0].stages : kStages;
  const uint32_t stage_bytes = EPI == kFew ? l.a[0].stage_bytes : kStageBytes;
  const uint32_t q_box = EPI == kFew ? (uint32_t)l.a[0].q_tile / 2 * 128 : kBoxBytes;      // bytes of one k-block of Q

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
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
      for (int i = 0, which, t; ok && next_tile<EPI>(l, pair, pairs, i, which, t); ++i) {
        const HeadArgs& a = l.a[is_store(EPI) ? which : 0];
        const CUtensorMap* map_p = &l.p[is_store(EPI) ? which : 0];
        const CUtensorMap* map_q = &l.q[is_store(EPI) ? which : 0];
        const bool p_mn = is_store(EPI) ? a.p_mn != 0 : P_MN, q_mn = is_store(EPI) ? a.q_mn != 0 : Q_MN;
        int split, m0, n0, s0, s1;
        tile_origin(a, t, split, m0, n0);
        split_range(a, split, s0, s1);
        m0 += (int)rank * 128;
        n0 += (EPI == kFew ? (int)rank * a.q_tile / 2 : (int)rank * 128) + a.q_n0;
        for (int kt = s0; kt < s1; ++kt, ++it) {
          const int s = it % stages;
          if (!mbar_wait(&empty[s], ((it / stages) & 1) ^ 1, abort_flag, status)) { ok = false; break; }
          uint8_t* sp = smem + (size_t)s * stage_bytes;
          uint8_t* sq = sp + kSub * kBoxBytes;
          const int subs = min(kSub, a.kblocks - kt * kSub);
          if (rank == 0) mbar_expect_tx(&full[s], (uint32_t)subs * 2 * (kBoxBytes + q_box));   // both CTAs' bytes
          const uint32_t bar = lead_full + 8u * s;
#pragma unroll
          for (int j = 0; j < kSub; ++j) {
            if (j < subs) {
              const int k0 = (kt * kSub + j) * kHeadK;
              // an operand whose m (or n) is contiguous: boxes of 64 of them by 64 k
              if (p_mn) {
                tma_load_pair(sp + j * kBoxBytes, map_p, bar, m0, k0);
                tma_load_pair(sp + j * kBoxBytes + kBoxBytes / 2, map_p, bar, m0 + 64, k0);
              } else {
                tma_load_pair(sp + j * kBoxBytes, map_p, bar, k0, m0);
              }
              if (q_mn) {
                tma_load_pair(sq + j * kBoxBytes, map_q, bar, n0, a.q_k0 + k0);
                tma_load_pair(sq + j * kBoxBytes + kBoxBytes / 2, map_q, bar, n0 + 64, a.q_k0 + k0);
              } else {
                tma_load_pair(sq + j * q_box, map_q, bar, a.q_k0 + k0, n0);
              }
            }
          }
        }
      }
      // Copies in flight must land before shared memory is released; the leader sees both CTAs'.
      if (rank == 0) {
        for (uint32_t j = it > stages ? it - stages : 0; j < it; ++j) {
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(&full[j % stages], (j / stages) & 1) && global_ns() - t0 < 1000000ull) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, acc = 0;
      bool ok = true;
      const uint32_t smem0 = smem_u32(smem);
      for (int i = 0, which, t; ok && next_tile<EPI>(l, pair, pairs, i, which, t); ++i) {
        const HeadArgs& a = l.a[is_store(EPI) ? which : 0];
        const bool p_mn = is_store(EPI) ? a.p_mn != 0 : P_MN, q_mn = is_store(EPI) ? a.q_mn != 0 : Q_MN;
        const uint32_t idesc = idesc_bf16(kTile, EPI == kFew ? a.q_tile : kTile, p_mn, q_mn);
        const uint32_t step_p = p_mn ? 128 : 2, step_q = q_mn ? 128 : 2;      // 16 k, in units of 16 bytes
        const int kblocks = a.kblocks;
        int split, m0, n0, s0, s1;
        tile_origin(a, t, split, m0, n0);
        split_range(a, split, s0, s1);
        for (int c0 = s0, c1; c0 < s1 && ok; c0 = c1, ++acc) {
          c1 = c0 + min(chunk_of(EPI), s1 - c0);
          const uint32_t ab = acc & 1;
          if (!mbar_wait(&tempty[ab], ((acc >> 1) & 1) ^ 1, abort_flag, status)) { ok = false; break; }
          tcgen05_after_sync();
          const uint32_t d = tmem + ab * kTile;
          for (int kt = c0; kt < c1; ++kt, ++it) {
            const int s = it % stages;
            if (!mbar_wait(&full[s], (it / stages) & 1, abort_flag, status)) { ok = false; break; }
            tcgen05_after_sync();
            const uint32_t sp = smem0 + (uint32_t)s * stage_bytes, sq = sp + kSub * kBoxBytes;
            const int subs = min(kSub, kblocks - kt * kSub);
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
              if (j < subs) {
                const uint64_t dp = p_mn ? desc_mn_major(sp + j * kBoxBytes, kBoxBytes / 2) : desc_k_major(sp + j * kBoxBytes);
                const uint64_t dq = q_mn ? desc_mn_major(sq + j * kBoxBytes, kBoxBytes / 2) : desc_k_major(sq + j * q_box);
#pragma unroll
                for (int k = 0; k < kHeadK / 16; ++k)
                  umma_bf16_pair(d, dp + step_p * k, dq + step_q * k, idesc, (uint32_t)(kt > c0) | (uint32_t)((j | k) != 0));
              }
            }
            umma_commit_both(smem_u32(&empty[s]));
          }
          if (ok) umma_commit_both(smem_u32(&tfull[ab]));
        }
      }
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t lead_tempty = cluster_map(smem_u32(&tempty[0]), 0);
    uint8_t* patch = smem + (size_t)stages * stage_bytes + (warp - 2) * kPatchBytes;
    float unit = 1.f;
    if constexpr (is_grad(EPI)) {
      const HeadArgs& a = l.a[0];
      if (a.unit) unit = *a.unit;
      if (a.unit_out) {
        float* red = reinterpret_cast<float*>(smem + (size_t)stages * stage_bytes);        // the patches
        const float share = unit_share<kEpiWarps * 32>(a.grad_loss, a.labels, a.vocab, a.m, (int)threadIdx.x - 64);
        if (lane == 0) red[warp - 2] = share;
        asm volatile("bar.sync 1, %0;" ::"n"(kEpiWarps * 32) : "memory");
        unit = 0.f;
#pragma unroll
        for (int k = 0; k < kEpiWarps; ++k) unit = fmaxf(unit, red[k]);
        unit = unit_of(unit);
        asm volatile("bar.sync 1, %0;" ::"n"(kEpiWarps * 32) : "memory");
        if (blockIdx.x == 0 && threadIdx.x == 64) *a.unit_out = unit;
      }
      // under the first tile's main loop
      if (a.clean) copy_live_rows(a, (int)blockIdx.x * kEpiWarps + warp - 2, (int)gridDim.x * kEpiWarps);
    }
    uint32_t acc = 0;
    bool ok = true;
    for (int i = 0, which, t; ok && next_tile<EPI>(l, pair, pairs, i, which, t); ++i) {
      const HeadArgs& a = l.a[is_store(EPI) ? which : 0];
      int split, m0, n0, s0, s1;
      tile_origin(a, t, split, m0, n0);
      const int column = (n0 / kTile) * 2 + half;
      m0 += (int)rank * 128 + quad * 32;                  // this warp's rows and columns
      // The accumulator is the next product's as soon as all warps of the pair have read it.
      auto wait = [&]() {
        const bool got = mbar_wait(&tfull[acc & 1], (acc >> 1) & 1, abort_flag, status);
        ok = __all_sync(0xffffffffu, got);
        tcgen05_after_sync();
        return ok;
      };
      auto release = [&]() {
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) arrive_cluster(lead_tempty + 8u * (acc & 1));
        ++acc;
      };
      if constexpr (EPI == kStats) {
        float v[128];
#pragma unroll
        for (int j = 0; j < 128; ++j) v[j] = 0.f;
        split_range(a, split, s0, s1);
#pragma unroll 1
        for (int c = s0; c < s1; c += chunk_of(EPI)) {
          if (!wait()) break;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            uint32_t r[16];
            tmem_ld16(trow + (acc & 1) * kTile + half * 128 + k * 16, r);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[k * 16 + j] += __uint_as_float(r[j]);
          }
          release();
        }
        if (ok) stats_tile(a, v, m0 + lane, n0 + half * 128, column);
      } else if constexpr (EPI == kFew) {
        float v[kFewRows / 2];                            // every other 16 of the rows
#pragma unroll
        for (int j = 0; j < kFewRows / 2; ++j) v[j] = 0.f;
        split_range(a, split, s0, s1);
#pragma unroll 1
        for (int c = s0; c < s1; c += chunk_of(EPI)) {
          if (!wait()) break;
#pragma unroll
          for (int g = 0; g < kFewRows / 32; ++g) {
            if ((g * 2 + half) * 16 < a.q_tile) {
              uint32_t r[16];
              tmem_ld16(trow + (acc & 1) * kTile + (g * 2 + half) * 16, r);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 16; ++j) v[g * 16 + j] += __uint_as_float(r[j]);
            }
          }
          release();
        }
        if (ok) {
#pragma unroll
          for (int g = 0; g < kFewRows / 32; ++g)
            if ((g * 2 + half) * 16 < a.q_tile)
              few_tile(a, v + g * 16, reinterpret_cast<float*>(patch), m0, n0 + (g * 2 + half) * 16);
        }
      } else {
        split_range(a, split, s0, s1);
        const uint32_t at = trow + half * 128;
        if (!wait()) break;
        if constexpr (EPI == kGradLong || EPI == kStoreLong) {
          if (s1 - s0 > chunk_of(EPI)) {                  // added in registers, and put where the last chunk's sums were
            float v[128];
#pragma unroll
            for (int j = 0; j < 128; ++j) v[j] = 0.f;
#pragma unroll 1
            for (int c = s0;;) {
              add_sums(at + (acc & 1) * kTile, v);
              c += chunk_of(EPI);
              if (c >= s1) break;
              release();
              if (!wait()) break;
            }
            if (!ok) break;
            put_sums(at + (acc & 1) * kTile, v);
          }
        }
        const int rows = min(32, a.m - m0);
        const uint32_t taddr = at + (acc & 1) * kTile;
        n0 += half * 128;
        if constexpr (is_grad(EPI)) grad_tile(a, taddr, patch, m0, n0, rows, unit);
        if constexpr (is_store(EPI)) {
          unit = a.unit ? *a.unit : 1.f;
          if (a.out_fp32) store_tile<float>(a, taddr, patch, split, m0, n0, rows, unit);
          else store_tile<__nv_bfloat16>(a, taddr, patch, split, m0, n0, rows, unit);
        }
        release();
      }
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

// A row's largest logit and sum relative to it.
struct Softmax {
  float top = -INFINITY, sum = 0.f;
  __device__ __forceinline__ void add(float p_top, float p_sum) {
    const float here = fmaxf(top, p_top);
    // a part of -infinities alone has the sum 0 (NaN with a NaN among them)
    if (top != here && top != -INFINITY) sum *= expf(top - here);
    sum += p_top == here || p_top == -INFINITY ? p_sum : p_sum * expf(p_top - here);
    top = here;
  }
};

// The rows' parts joined: `each` rows per block (a power of two up to 32), 256 / each threads to a row.
__global__ void __launch_bounds__(256) head_join_kernel(const float2* part, int parts, const float* at_label, const int64_t* labels,
                                                        int64_t vocab, int rows, int each, float* loss, float* lse) {
  __shared__ float2 s[8][32];
  grid_wait();
  grid_trigger();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int row = (int)blockIdx.x * each + threadIdx.x % each;
  Softmax m;
  if (row < rows) {
#pragma unroll 4
    for (int k = threadIdx.x / each; k < parts; k += 256 / each) {
      const float2 p = __ldcg(part + (int64_t)k * rows + row);
      m.add(p.x, p.y);
    }
  }
  for (int o = each; o < 32; o *= 2) {
    const float top = __shfl_xor_sync(0xffffffffu, m.top, o), sum = __shfl_xor_sync(0xffffffffu, m.sum, o);
    m.add(top, sum);
  }
  s[warp][lane] = make_float2(m.top, m.sum);
  __syncthreads();
  if (warp == 0 && lane < each && row < rows) {
#pragma unroll
    for (int k = 1; k < 8; ++k) m.add(s[k][lane].x, s[k][lane].y);
    const float rest = logf(m.sum);        // at least 0
    const int64_t label = labels[row];
    lse[row] = m.top + rest;
    // not lse - logit, whose rounding can leave less than 0
    loss[row] = label >= 0 && label < vocab ? (m.top - at_label[row]) + rest : 0.f;
  }
}

__global__ void __launch_bounds__(1024) head_unit_kernel(const float* grad_loss, const int64_t* labels, int64_t vocab, int rows,
                                                         float* unit) {
  __shared__ float red[32];
  grid_wait();
  grid_trigger();
  const float share = unit_share<1024>(grad_loss, labels, vocab, rows, threadIdx.x);
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = share;
  __syncthreads();
  if (threadIdx.x < 32) {
    const float top = group_top(red[threadIdx.x]);
    if (threadIdx.x == 0) *unit = unit_of(top);
  }
}

// A copy of an operand whose rows do not start on 16 bytes, which the copies into shared memory need: eight elements per thread.
__global__ void __launch_bounds__(256) head_copy_kernel(const uint16_t* p, int64_t ld, int64_t rows, int cols, uint16_t* out,
                                                        int64_t ld_out) {
  grid_wait();
  grid_trigger();
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, octs = ld_out / 8, row = at / octs;
  if (row >= rows) return;
  const int c = (int)(at - row * octs) * 8;
  p += row * ld + c;
  uint4 v;
  if (c + 8 <= cols && ((uintptr_t)p & 2) == 0) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
    v = make_uint4(w[0], w[1], w[2], w[3]);
  } else if (c + 8 <= cols) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p + 1);
    const uint32_t e0 = p[0], w0 = w[0], w1 = w[1], w2 = w[2], e7 = p[7];
    v = make_uint4(e0 | w0 << 16, w0 >> 16 | w1 << 16, w1 >> 16 | w2 << 16, w2 >> 16 | e7 << 16);
  } else {
    uint32_t e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) e[k] = c + k < cols ? p[k] : 0;
    v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
  }
  *reinterpret_cast<uint4*>(out + row * ld_out + c) = v;
}

// grad_x from the parts of its sums.
__global__ void __launch_bounds__(256) head_sum_kernel(const float* part, int parts, int64_t stride, int rows, int cols,
                                                       int64_t ld_part, const float* unit, __nv_bfloat16* out, int64_t ld_out) {
  grid_wait();
  grid_trigger();
  const float c = *unit;
  const int chunks = (cols + 255) / 256;
  const int64_t row = blockIdx.x / (unsigned)chunks;
  const int col = (int)(blockIdx.x % (unsigned)chunks) * 256 + threadIdx.x;
  if (col >= cols) return;
  float sum = 0.f;
  for (int k = 0; k < parts; ++k) sum += __ldcg(part + k * stride + row * ld_part + col);
  out[row * ld_out + col] = __float2bfloat16_rn(sum * c);
}

// Map over a row-major rows x cols bf16 matrix, boxes of box_rows x 64; what lies outside reads as zero.
bool make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  Q8EncodeFn encode = q8_encode_fn();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {kHeadK, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Operand {
  const void* p;
  int64_t rows, cols, ld;          // as stored
  bool mn;                         // m (n) contiguous
};

// Fills in product i of a launch.
template <int EPI>
int set_product(HeadLaunch& l, int i, const Operand& p, const Operand& q, HeadArgs a, int64_t k) {
  a.status = q8_status_word();
  if (!a.status) return PRM_ERR_CUDA;
  if constexpr (EPI == kFew) {
    a.q_tile = (int)ceil_to(a.n, 16);
    a.stage_bytes = kSub * (kBoxBytes + (uint32_t)a.q_tile / 2 * 128);
    a.stages = std::min<int>(kMaxStages, (int)(kStages * kStageBytes / a.stage_bytes));
  }
  a.p_mn = p.mn;
  a.q_mn = q.mn;
  a.kblocks = (int)((k + kHeadK - 1) / kHeadK);
  a.m_tiles = (a.m + kTile - 1) / kTile;
  a.n_tiles = (a.n + kTile - 1) / kTile;
  if ((int64_t)a.m_tiles * a.n_tiles * a.split > 0x3fffffffLL) return PRM_ERR_SHAPE;
  a.tiles = a.m_tiles * a.n_tiles * a.split;
  // As many m-tiles as keep their rows of P within 32 MB of the L2, at least 8 (a ninth of a wave).
  const int64_t fit = ((int64_t)32 << 20) / ((int64_t)kTile * a.kblocks * 128);
  a.band = (int)std::min<int64_t>(a.m_tiles, std::max<int64_t>(8, fit));
  l.a[i] = a;
  return make_map(&l.p[i], p.p, p.rows, p.cols, p.ld, p.mn ? 64 : 128) &&
                 make_map(&l.q[i], q.p, q.rows, q.cols, q.ld, EPI == kFew ? a.q_tile / 2 : q.mn ? 64 : 128)
             ? PRM_OK
             : PRM_ERR_CUDA;
}
template <int EPI, bool P_MN, bool Q_MN>
int launch_products(const HeadLaunch& l, cudaStream_t stream) {
  static PerDeviceOnce once;
  static int resident[64];
  int dev;
  if (once.need(&dev)) {
    if (dev < 0) return PRM_ERR_CUDA;
    const cudaError_t e = cudaFuncSetAttribute(head_kernel<EPI, P_MN, Q_MN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)kSmemBytes);
    if (e != cudaSuccess) return q8_code(e);
    const int n = q8_resident_clusters(head_kernel<EPI, P_MN, Q_MN>, kThreads, kSmemBytes, 2);
    if (n < 1) return PRM_ERR_CUDA;
    resident[dev] = n;
    once.mark(dev);
  }
  return q8_code(launch_after(head_kernel<EPI, P_MN, Q_MN>, 2u * (unsigned)std::min(l.a[0].tiles + l.a[1].tiles, resident[dev]),
                              kThreads, kSmemBytes, stream, 2, l));
}
template <int EPI, bool P_MN, bool Q_MN>
int launch_head(const Operand& p, const Operand& q, const HeadArgs& a, int64_t k, cudaStream_t stream) {
  HeadLaunch l = {};
  const int code = set_product<EPI>(l, 0, p, q, a, k);
  return code == PRM_OK ? launch_products<EPI, P_MN, Q_MN>(l, stream) : code;
}
// Stages of a tile at most; and how long it takes, in stages: its main loop, or its epilogue where that is longer (5 stages).
inline int tile_stages(const HeadArgs& a) { return ((a.kblocks + kSub - 1) / kSub + a.split - 1) / a.split; }
inline int tile_cost(const HeadArgs& a) { return std::max(5, (a.kblocks + kSub - 1) / kSub / std::max(1, a.split)); }
int launch_few(const Operand& x, const Operand& w, const HeadArgs& a, int64_t d, cudaStream_t stream) {
  return w.mn ? launch_head<kFew, true, false>(w, x, a, d, stream) : launch_head<kFew, false, false>(w, x, a, d, stream);
}
template <int EPI>
int launch_logits(const Operand& x, const Operand& w, const HeadArgs& a, int64_t d, cudaStream_t stream) {
  return w.mn ? launch_head<EPI, false, true>(x, w, a, d, stream) : launch_head<EPI, false, false>(x, w, a, d, stream);
}

// ------------------------------------------------------------------ sizes

// Forward: what is left of each row, and rows whose parts fit 128 MB are taken together.
int64_t stats_parts(int64_t n, int64_t vocab) { return (n <= kFewRows ? 8 : 2) * ((vocab + kTile - 1) / kTile); }
int64_t stats_rows(int64_t n, int64_t vocab) {
  const int64_t parts = stats_parts(n, vocab);
  return std::min(n, std::max<int64_t>(2048, ((int64_t)128 << 20) / (8 * parts) / kTile * kTile));
}

// Sums as long as 2^27 leave a tile in its main loop for less than a second, half of what a wait is given.
bool sizes_ok(int64_t n, int64_t d, int64_t vocab) {
  const int64_t most = (int64_t)1 << 27;
  return n >= 0 && d >= 1 && vocab >= 1 && n <= most && d <= most && vocab <= most;
}
// Whether a matrix can be read at all: PRM_OK, or why not.
int operand_code(const void* p, int64_t ld, int64_t cols) {
  if (!p) return PRM_ERR_ARG;
  if (ld < cols || ld >= ((int64_t)1 << 38)) return PRM_ERR_SHAPE;
  return (uintptr_t)p % 2 == 0 ? PRM_OK : PRM_ERR_ALIGN;
}
bool operand_aligned(const void* p, int64_t ld) { return aligned16(p) && ld % 8 == 0; }
size_t copy_bytes(int64_t rows, int64_t cols) { return (size_t)ceil_to(rows * ceil_to(cols, 8) * 2, 256); }
// Puts a copy of an operand that is not aligned at `tail` and moves both on.
int place(const void*& p, int64_t& ld, int64_t rows, int64_t cols, char*& tail, cudaStream_t stream) {
  if (operand_aligned(p, ld)) return PRM_OK;
  const int64_t wide = ceil_to(cols, 8), blocks = (rows * (wide / 8) + 255) / 256;
  if (blocks > 0x7fffffffLL) return PRM_ERR_SHAPE;
  const int code = q8_code(launch_after(head_copy_kernel, (unsigned)blocks, 256, 0, stream, 0, (const uint16_t*)p, ld, rows,
                                        (int)cols, (uint16_t*)tail, wide));
  p = tail;
  ld = wide;
  tail += copy_bytes(rows, cols);
  return code;
}

}  // namespace
}  // namespace prm

using namespace prm;

extern "C" size_t prm_head_loss_copy_bytes(int64_t rows, int64_t cols) {
  return rows < 1 || cols < 1 ? 0 : copy_bytes(rows, cols);
}

extern "C" size_t prm_head_loss_scratch_bytes(int64_t n, int64_t d, int64_t vocab) {
  if (n < 1 || !sizes_ok(n, d, vocab)) return 0;
  return (size_t)ceil_to((int64_t)stats_rows(n, vocab) * (stats_parts(n, vocab) * 8 + 4), 256);
}

extern "C" int prm_head_loss(const void* x, int64_t ld_x, const void* weight, int64_t ld_weight, int weight_transposed,
                             const int64_t* labels, int64_t n, int64_t d, int64_t vocab, float* loss_out, float* lse_out,
                             void* scratch, size_t scratch_bytes, void* cuda_stream) {
  if (!sizes_ok(n, d, vocab)) return PRM_ERR_SHAPE;
  if (n == 0) return PRM_OK;
  if (!labels || !loss_out || !lse_out || !scratch) return PRM_ERR_ARG;
  int code = operand_code(x, ld_x, d);
  if (code == PRM_OK) code = operand_code(weight, ld_weight, weight_transposed ? d : vocab);
  if (code != PRM_OK) return code;
  if (((uintptr_t)loss_out | (uintptr_t)lse_out) % 4 != 0 || (uintptr_t)labels % 8 != 0 || !aligned16(scratch))
    return PRM_ERR_ALIGN;
  const int64_t w_rows = weight_transposed ? vocab : d, w_cols = weight_transposed ? d : vocab;
  const size_t base = prm_head_loss_scratch_bytes(n, d, vocab);
  if (scratch_bytes < base + (operand_aligned(x, ld_x) ? 0 : copy_bytes(n, d)) +
                          (operand_aligned(weight, ld_weight) ? 0 : copy_bytes(w_rows, w_cols)))
    return PRM_ERR_WORKSPACE;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  char* tail = (char*)scratch + base;
  code = place(x, ld_x, n, d, tail, stream);
  if (code == PRM_OK) code = place(weight, ld_weight, w_rows, w_cols, tail, stream);
  if (code != PRM_OK) return code;
  const Operand w = {weight, w_rows, w_cols, ld_weight, !weight_transposed};
  const int64_t step = stats_rows(n, vocab);
  const int parts = (int)stats_parts(n, vocab);
  for (int64_t r = 0; r < n; r += step) {
    const int64_t rows = std::min(step, n - r);
    HeadArgs a = {};
    const bool few = n <= kFewRows;
    a.m = (int)(few ? vocab : rows);
    a.n = (int)(few ? rows : vocab);
    a.split = 1;
    a.labels = labels + r;
    a.vocab = vocab;
    a.part = (float2*)scratch;
    a.at_label = (float*)(a.part + (size_t)parts * rows);
    const Operand xr = {(const __nv_bfloat16*)x + r * ld_x, rows, d, ld_x, false};
    // in the few rows' form W is the left operand, whose m is W's column
    const Operand wl = {weight, w.rows, w.cols, ld_weight, !weight_transposed};
    code = few ? launch_few(xr, wl, a, d, stream) : launch_logits<kStats>(xr, w, a, d, stream);
    if (code != PRM_OK) return code;
    int each = 1;                          // few rows: more threads to each, on all SMs
    while (each < 32 && rows > (int64_t)each * 148) each *= 2;
    code = q8_code(launch_after(head_join_kernel, (unsigned)((rows + each - 1) / each), 256, 0, stream, 0, a.part, parts,
                                a.at_label, a.labels, vocab, (int)rows, each, loss_out + r, lse_out + r));
    if (code != PRM_OK) return code;
  }
  return PRM_OK;
}

extern "C" size_t prm_head_loss_backward_scratch_bytes(int64_t n, int64_t d, int64_t vocab) {
  if (n < 1 || !sizes_ok(n, d, vocab)) return 0;
  const HeadGradPlan p = head_grad_plan(n, d, vocab);
  return 256 + p.g_bytes + (size_t)ceil_to((int64_t)p.part_bytes, 256) + copy_bytes(n, d);
}

extern "C" int prm_head_loss_backward(const float* grad_loss, const void* x, int64_t ld_x, const void* weight,
                                      int64_t ld_weight, int weight_transposed, const int64_t* labels, const float* lse,
                                      int64_t n, int64_t d, int64_t vocab, void* grad_x, int64_t ld_grad_x,
                                      void* grad_weight, int64_t ld_grad_weight, void* scratch, size_t scratch_bytes,
                                      void* cuda_stream) {
  if (!sizes_ok(n, d, vocab)) return PRM_ERR_SHAPE;
  const int64_t w_rows = weight_transposed ? vocab : d, w_cols = weight_transposed ? d : vocab;
  if (grad_x && (ld_grad_x < d || ld_grad_x > ((int64_t)1 << 40))) return PRM_ERR_SHAPE;
  if (grad_weight && (ld_grad_weight < w_cols || ld_grad_weight > ((int64_t)1 << 40))) return PRM_ERR_SHAPE;
  if (((uintptr_t)grad_x | (uintptr_t)grad_weight) % 2 != 0) return PRM_ERR_ALIGN;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (n == 0)                             // an empty sum
    return !grad_weight ? PRM_OK : q8_code(cudaMemset2DAsync(grad_weight, (size_t)ld_grad_weight * 2, 0, (size_t)w_cols * 2,
                                                             (size_t)w_rows, stream));
  if (!grad_x && !grad_weight) return PRM_OK;
  if (!grad_loss || !labels || !lse || !scratch) return PRM_ERR_ARG;
  int code = operand_code(x, ld_x, d);
  if (code == PRM_OK) code = operand_code(weight, ld_weight, w_cols);
  if (code != PRM_OK) return code;
  if (((uintptr_t)grad_loss | (uintptr_t)lse) % 4 != 0 || (uintptr_t)labels % 8 != 0 || ((uintptr_t)scratch & 255) != 0)
    return PRM_ERR_ALIGN;
  // x is copied for grad_weight only
  const size_t kept = grad_weight ? copy_bytes(n, d) : 0, base = prm_head_loss_backward_scratch_bytes(n, d, vocab) - copy_bytes(n, d) + kept;
  if (scratch_bytes < base + (operand_aligned(x, ld_x) ? 0 : copy_bytes(n, d)) +
                          (operand_aligned(weight, ld_weight) ? 0 : copy_bytes(w_rows, w_cols)))
    return PRM_ERR_WORKSPACE;
  char* tail = (char*)scratch + base;
  code = place(x, ld_x, n, d, tail, stream);
  if (code == PRM_OK) code = place(weight, ld_weight, w_rows, w_cols, tail, stream);
  const HeadGradPlan plan = head_grad_plan(n, d, vocab);
  float* unit = (float*)scratch;
  __nv_bfloat16* g = (__nv_bfloat16*)((char*)scratch + 256);
  float* part = (float*)((char*)g + plan.g_bytes);
  __nv_bfloat16* clean = (__nv_bfloat16*)((char*)scratch + base - kept);
  const int64_t ld_clean = ceil_to(d, 8);
  const Operand w = {weight, w_rows, w_cols, ld_weight, !weight_transposed};
  if (code == PRM_OK && n > kUnitRows) code = q8_code(launch_after(head_unit_kernel, 1u, 1024, 0, stream, 0, grad_loss, labels, vocab, (int)n, unit));
  const bool parted = plan.part_bytes > 0;
  for (int64_t v0 = 0; v0 < vocab && code == PRM_OK; v0 += plan.piece) {
    const int64_t wide = std::min(plan.piece, vocab - v0);
    HeadArgs a = {};
    a.m = (int)n;
    a.n = (int)wide;
    a.q_n0 = (int)v0;
    a.split = 1;
    a.labels = labels;
    a.vocab = vocab;
    a.lse = lse;
    a.grad_loss = grad_loss;
    a.g = g;
    a.ld_g = plan.ld_g;
    a.unit = n > kUnitRows || v0 > 0 ? unit : nullptr;
    a.unit_out = a.unit ? nullptr : unit;
    a.x = (const __nv_bfloat16*)x;
    a.ld_x = ld_x;
    a.clean = grad_weight && v0 == 0 ? clean : nullptr;
    a.ld_clean = ld_clean;
    a.d = (int)d;
    const Operand xp = {x, n, d, ld_x, false};
    code = d <= kLogitChunk * kHeadStage ? launch_logits<kGrad>(xp, w, a, d, stream) : launch_logits<kGradLong>(xp, w, a, d, stream);
    HeadLaunch l = {};                     // the two products that read G: one launch
    int products = 0;
    if (code == PRM_OK && grad_x) {
      HeadArgs b = {};
      b.m = (int)n;
      b.n = (int)d;
      b.q_k0 = (int)v0;
      b.split = head_grad_split(plan, wide);
      b.unit = parted ? nullptr : unit;
      b.out = parted ? (void*)part : grad_x;
      b.ld_out = parted ? plan.ld_part : ld_grad_x;
      b.split_stride = n * plan.ld_part;
      b.out_fp32 = parted;
      b.accumulate = v0 > 0;
      const Operand gp = {g, n, wide, plan.ld_g, false}, wq = {weight, w_rows, w_cols, ld_weight, weight_transposed != 0};
      code = set_product<kStore>(l, products++, gp, wq, b, wide);
    }
    if (code == PRM_OK && grad_weight) {
      HeadArgs b = {};
      b.split = 1;
      b.unit = unit;
      b.ld_out = ld_grad_weight;
      const Operand gt = {g, n, wide, plan.ld_g, true}, xt = {clean, n, d, ld_clean, true};
      if (weight_transposed) {
        b.m = (int)wide;
        b.n = (int)d;
        b.out = (__nv_bfloat16*)grad_weight + v0 * ld_grad_weight;
        code = set_product<kStore>(l, products++, gt, xt, b, n);
      } else {
        b.m = (int)d;
        b.n = (int)wide;
        b.out = (__nv_bfloat16*)grad_weight + v0;
        code = set_product<kStore>(l, products++, xt, gt, b, n);
      }
    }
    if (code == PRM_OK) {
      if (products == 2) l.extra = tile_cost(l.a[0]) / tile_cost(l.a[1]);
      code = std::max(tile_stages(l.a[0]), products == 2 ? tile_stages(l.a[1]) : 0) > kStoreLongest
                 ? launch_products<kStoreLong, false, false>(l, stream)
                 : launch_products<kStore, false, false>(l, stream);
    }
  }
  if (code == PRM_OK && grad_x && parted) {
    const int64_t blocks = n * ((d + 255) / 256);
    if (blocks > 0x7fffffffLL) return PRM_ERR_SHAPE;
    code = q8_code(launch_after(head_sum_kernel, (unsigned)blocks, 256, 0, stream, 0, (const float*)part, plan.split,
                                n * plan.ld_part, (int)n, (int)d, plan.ld_part, (const float*)unit, (__nv_bfloat16*)grad_x,
                                ld_grad_x));
  }
  return code;
}
