// Cross entropy of given tokens under the output projection, and its gradients, on
// the tensor cores; the N x V logits are never stored.
//
//   x[r, v] = hidden[r] . weight[v],  lse[r] = ln sum_v e^x,  loss[r] = lse[r] - x[r, t_r]
//   g[r, v] = dloss[r] (e^(x - lse[r]) - [v = t_r])
//   d_hidden = g weight,   d_weight = g^T hidden
//
// Rows without a target (outside [0, V)) are not scored: the first launch copies the
// hidden states of the others, in their order, to the workspace (n rows, then rows of
// zeros to a multiple of 128), so the products take time for scored rows alone -- of a
// masked diffusion batch a quarter, say -- and their number stays on the GPU.
//
// Four products run through one persistent kernel, a CTA an SM, 128 x bn output tiles
// (bn up to 256), K steps of 64 through a ring of four stages of 48 KB:
//   stats  x = H W^T     per row and part of the vocabulary: maximum, sum of e^(x - m),
//                        and the target's logit; loss_combine_kernel joins the parts
//   grad   x = H W^T     g of one piece of the vocabulary, rounded to bf16, to the workspace
//   dw     g^T H         a piece of d_weight, bf16
//   dh     g W           fp32 sums over the piece, added to those of the pieces before it;
//                        split over K where there are too few tiles for every SM
// g is rounded to bf16 because the tensor cores take it so: every term of d_hidden and
// d_weight is off by at most 2^-8 relative, as the result is by its own rounding to bf16;
// all sums are fp32. Warp 0 loads by TMA, warp 1 issues tcgen05.mma (both operands in
// shared memory, K-major or MN-major as their matrix lies in memory, so nothing is
// transposed), warps 4-7 read the fp32 accumulators (two, so a tile's epilogue runs
// under the next one's K loop) and write their tiles through shared memory by TMA.
// Every wait is bounded; on expiry the kernel sets DLM_DEVERR_TIMEOUT, drains and exits.
#include <cuda.h>
#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"
#include "dlm_tmap.h"

namespace dlm {
namespace {

constexpr int kBM = 128;          // rows of an output tile = TMEM lanes
constexpr int kBK = 64;           // K of a stage: 128 bytes of bf16
constexpr int kMaxBN = 256;
constexpr int kStages = 4;
constexpr int kThreads = 256;     // warp 0 TMA, warp 1 MMA, warps 4-7 epilogue
constexpr int kEpiWarp0 = 4;
constexpr int kABytes = kBM * kBK * 2;
constexpr int kBBytes = kMaxBN * kBK * 2;
constexpr int kBoxBytes = 64 * 128;          // an MN-major box: 64 K rows of 64 columns
constexpr uint32_t kTmemCols = 2 * kMaxBN;   // two accumulators
constexpr float kLog2e = 1.4426950408889634f;

enum Mode { kStats, kGrad, kDw, kDh };

struct Smem {
  alignas(1024) uint8_t a[kStages][kABytes];
  alignas(1024) uint8_t b[kStages][kBBytes];
  alignas(1024) uint8_t out[4][2][32 * 128];  // per epilogue warp, two buffers of 32 rows x 128 bytes
  uint64_t full[kStages];   // stage loaded            (TMA -> MMA)
  uint64_t empty[kStages];  // stage read by its MMAs  (MMA -> TMA)
  uint64_t acc_full[2];     // accumulator complete    (MMA -> epilogue)
  uint64_t acc_empty[2];    // accumulator read out    (epilogue -> MMA)
  uint64_t done;            // every MMA completed     (teardown)
  uint32_t tmem_base;
  int abort;
};
constexpr size_t kSmemBytes = sizeof(Smem) + 1024;
static_assert(kSmemBytes <= 227 * 1024, "shared memory of a CTA");

// What the first launch leaves for the others.
struct Plan {
  int n;       // scored rows
  int splits;  // K splits of dh
};

struct Params {
  const Plan* plan;
  int V;
  int kblocks;          // stats, grad: K steps (of d);  dh: of the piece
  int bn;               // columns of a tile
  int tiles;            // stats, grad: vocabulary tiles;  dw, dh: tiles of d
  int parts;            // stats: parts of the vocabulary;  dw: tiles of the piece's rows
  int v0;               // first vocabulary column of the piece
  int a_rows;           // stats: rows of the hidden box
  int add;              // dh: add to what the pieces before left
  int rows_out, cols_out;  // dw, dh: extents of what is written
  const int* target;    // of each scored row
  const float* lse2;    // lse log2(e)
  const float* dloss;
  float2* part;         // stats: (maximum, sum) [part][row]
  float* x_target;      // stats: the target's logit
  int* err;
  uint64_t wait_ns;
};

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* err, uint64_t budget_ns) {
  const bool ok = mbar_wait_for(bar, parity, abort, err, budget_ns);
  return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ void tma_store_2d(const void* tmap, const void* src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(smem_u32(src)), "r"(c0), "r"(c1)
               : "memory");
}

// fp32 addition of a box to what is there.
__device__ __forceinline__ void tma_add_2d(const void* tmap, const void* src, int c0, int c1) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(smem_u32(src)), "r"(c0), "r"(c1)
               : "memory");
}

// One output tile and its K steps [k0, k1). m, n: its row and column tiles.
struct Tile {
  int m, n, k0, k1, split;
};

// The work of a launch: items, each a run of tiles [t0, t1) (one tile but for stats).
template <int kMode>
struct Work {
  int items, row_blocks, k, splits;

  __device__ Work(const Params& p) {
    const int n = p.plan->n;
    row_blocks = (n + kBM - 1) / kBM;
    splits = p.plan->splits;
    k = kMode == kDw ? (n + kBK - 1) / kBK : p.kblocks;
    items = kMode == kStats  ? p.parts * row_blocks
            : kMode == kGrad ? p.tiles * row_blocks
            : kMode == kDw   ? p.parts * p.tiles
                             : splits * row_blocks * p.tiles;
  }
  __device__ __forceinline__ int first(const Params& p, int item) const {
    return kMode == kStats ? static_cast<int>(static_cast<long long>(p.tiles) * (item / row_blocks) / p.parts) : 0;
  }
  __device__ __forceinline__ int last(const Params& p, int item) const {
    return kMode == kStats ? static_cast<int>(static_cast<long long>(p.tiles) * (item / row_blocks + 1) / p.parts) : 1;
  }
  // Items that run at the same time share vocabulary tiles (stats, grad: the row block
  // changes first) or the rows of g (dw, dh: the tile of d changes first).
  __device__ __forceinline__ Tile tile(const Params& p, int item, int t) const {
    if (kMode == kStats) return {item % row_blocks, t, 0, k, 0};
    if (kMode == kGrad) return {item % row_blocks, item / row_blocks, 0, k, 0};
    if (kMode == kDw) return {item / p.tiles, item % p.tiles, 0, k, 0};
    const int per = row_blocks * p.tiles, split = item / per, rest = item % per;
    return {rest / p.tiles, rest % p.tiles, static_cast<int>(static_cast<long long>(k) * split / splits),
            static_cast<int>(static_cast<long long>(k) * (split + 1) / splits), split};
  }
};

// ma, mb: the operands' maps; mo: the map written (none for stats).
template <int kMode>
__global__ void __launch_bounds__(kThreads, 1)
    loss_product_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
                        const __grid_constant__ CUtensorMap mo, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.acc_full[i], 1);
      mbar_init(&sm.acc_empty[i], 128);
    }
    mbar_init(&sm.done, 1);
    sm.abort = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  volatile int* abort = &sm.abort;
  wait_for_previous();
  const Work<kMode> work(p);
  const int boxes = p.bn / 64;  // MN-major boxes of B

  if (warp == 0) {
    // ================================================================ TMA producer
    if (lane == 0) {
      prefetch_tmap(&ma);
      prefetch_tmap(&mb);
    }
    const uint32_t stage_bytes = (kMode == kStats ? p.a_rows * 128 : kABytes) + p.bn * 128;
    int fill = 0;
    bool ok = true;
    for (int item = blockIdx.x; ok && item < work.items; item += gridDim.x) {
      const int t1 = work.last(p, item);
      for (int t = work.first(p, item); ok && t < t1; ++t) {
        const Tile tl = work.tile(p, item, t);
        for (int kb = tl.k0; kb < tl.k1; ++kb, ++fill) {
          const int st = fill % kStages;
          if (fill >= kStages && !warp_wait(&sm.empty[st], ((fill / kStages) - 1) & 1, abort, p.err, p.wait_ns)) {
            ok = false;
            break;
          }
          if (lane == 0) {
            mbar_arrive_expect_tx(&sm.full[st], stage_bytes);
            if (kMode == kStats || kMode == kGrad) {
              tma_load_2d(sm.a[st], &ma, &sm.full[st], kb * kBK, tl.m * kBM);
              tma_load_2d(sm.b[st], &mb, &sm.full[st], kb * kBK, p.v0 + tl.n * p.bn);
            } else if (kMode == kDw) {
              for (int j = 0; j < 2; ++j)
                tma_load_2d(sm.a[st] + j * kBoxBytes, &ma, &sm.full[st], tl.m * kBM + 64 * j, kb * kBK);
              for (int j = 0; j < boxes; ++j)
                tma_load_2d(sm.b[st] + j * kBoxBytes, &mb, &sm.full[st], tl.n * p.bn + 64 * j, kb * kBK);
            } else {
              tma_load_2d(sm.a[st], &ma, &sm.full[st], kb * kBK, tl.m * kBM);
              for (int j = 0; j < boxes; ++j)
                tma_load_2d(sm.b[st] + j * kBoxBytes, &mb, &sm.full[st], tl.n * p.bn + 64 * j, p.v0 + kb * kBK);
            }
          }
        }
      }
    }
    // Teardown: every copy issued lands before the block exits.
    if (lane == 0) {
      for (int s = 0; s < kStages; ++s) {
        const int n_s = fill > s ? (fill - s + kStages - 1) / kStages : 0;
        if (n_s) mbar_drain(&sm.full[s], (n_s - 1) & 1);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ================================================================ MMA issuer
    constexpr bool a_mn = kMode == kDw, b_mn = kMode == kDw || kMode == kDh;
    // A step of 16 in K: 32 bytes of each row (K-major), or 16 rows of 128 bytes (MN-major).
    constexpr uint32_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;
    const uint32_t idesc = idesc_bf16_f32(kBM, p.bn, a_mn, b_mn);
    const uint64_t a_desc0 = sdesc_sw128(smem_u32(sm.a[0]), a_mn ? kBoxBytes : 16, 1024);
    const uint64_t b_desc0 = sdesc_sw128(smem_u32(sm.b[0]), b_mn ? kBoxBytes : 16, 1024);
    int fill = 0, tile = 0;
    bool ok = true;
    for (int item = blockIdx.x; ok && item < work.items; item += gridDim.x) {
      const int t1 = work.last(p, item);
      for (int t = work.first(p, item); ok && t < t1; ++t, ++tile) {
        const Tile tl = work.tile(p, item, t);
        const int acc = tile & 1;
        // The accumulator's previous tile (tile - 2) must have been read out.
        if (tile >= 2 && !warp_wait(&sm.acc_empty[acc], ((tile >> 1) - 1) & 1, abort, p.err, p.wait_ns)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t d_tmem = tmem + acc * kMaxBN;
        for (int kb = tl.k0; kb < tl.k1; ++kb, ++fill) {
          const int st = fill % kStages;
          if (!warp_wait(&sm.full[st], (fill / kStages) & 1, abort, p.err, p.wait_ns)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t a_desc = a_desc0 + static_cast<uint32_t>(st) * (kABytes >> 4);
          const uint64_t b_desc = b_desc0 + static_cast<uint32_t>(st) * (kBBytes >> 4);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk)
            mma_ss_elect(d_tmem, a_desc + kk * a_step, b_desc + kk * b_step, idesc, (kb > tl.k0 || kk > 0) ? 1u : 0u);
          mma_commit_elect(&sm.empty[st]);
        }
        if (!ok) break;
        mma_commit_elect(&sm.acc_full[acc]);
      }
    }
    mma_commit_elect(&sm.done);
    mbar_drain(&sm.done, 0);
    __syncwarp();
  } else if (warp >= kEpiWarp0) {
    // ================================================================ epilogue
    const int qw = warp - kEpiWarp0;                 // TMEM lanes 32 qw .. 32 qw + 31
    const int t_row = qw * 32 + lane;                // row within the tile
    const uint32_t lane_base = static_cast<uint32_t>(qw * 32) << 16;
    int tile = 0, chunk = 0;
    bool ok = true;
    for (int item = blockIdx.x; ok && item < work.items; item += gridDim.x) {
      const int t1 = work.last(p, item);
      float m = -INFINITY, s = 0.f;  // stats: over the item's tiles
      int target = -1;
      float lse2 = 0.f, dloss = 0.f;
      if (kMode == kStats || kMode == kGrad) {
        const int row = (item % work.row_blocks) * kBM + t_row;
        target = p.target[row];
        if (kMode == kGrad) {
          lse2 = p.lse2[row];
          dloss = p.dloss[row];
        }
      }
      for (int t = work.first(p, item); t < t1; ++t, ++tile) {
        const Tile tl = work.tile(p, item, t);
        const int acc = tile & 1;
        if (!warp_wait(&sm.acc_full[acc], (tile >> 1) & 1, abort, p.err, p.wait_ns)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t base = tmem + lane_base + acc * kMaxBN;
        const int row = tl.m * kBM + t_row;
        float ts = 0.f;  // stats: this tile's terms, relative to m
#pragma unroll 1
        for (int c = 0; c < p.bn / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(base + 32 * c, v);
          tmem_wait_ld();
          if (c == p.bn / 32 - 1) {
            tc_fence_before();
            mbar_arrive(&sm.acc_empty[acc]);  // every column of the accumulator has been read
          }
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(v[e]);
          if (kMode == kStats) {
            const int col0 = tl.n * p.bn + 32 * c;
            if (static_cast<unsigned>(target - col0) < 32u) {
              float xt = x[0];
#pragma unroll
              for (int e = 1; e < 32; ++e)
                if (target - col0 == e) xt = x[e];
              p.x_target[row] = xt;
            }
            if (col0 + 32 > p.V) {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (col0 + e >= p.V) x[e] = -INFINITY;
            }
            float cm0 = fmaxf(x[0], x[1]), cm1 = fmaxf(x[2], x[3]);
#pragma unroll
            for (int e = 4; e < 32; e += 4) {
              cm0 = fmax3(cm0, x[e], x[e + 1]);
              cm1 = fmax3(cm1, x[e + 2], x[e + 3]);
            }
            const float cm = fmaxf(cm0, cm1);
            if (cm > m) {
              const float a = m == -INFINITY ? 1.f : ex2_approx((m - cm) * kLog2e);  // nothing, or a NaN, yet
              s *= a;
              ts *= a;
              m = cm;
            }
            const float ml = m == -INFINITY ? 0.f : m * kLog2e;
            const float2 k2 = make_float2(kLog2e, kLog2e), n2 = make_float2(-ml, -ml);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 y = ffma2(make_float2(x[e], x[e + 1]), k2, n2);
              sum = fadd2(sum, make_float2(ex2_approx(y.x), ex2_approx(y.y)));
            }
            ts += sum.x + sum.y;
          } else {
            if (kMode == kGrad) {
              const int col0 = p.v0 + tl.n * p.bn + 32 * c;
              const float2 k2 = make_float2(kLog2e, kLog2e), n2 = make_float2(-lse2, -lse2);
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                const float2 y = ffma2(make_float2(x[e], x[e + 1]), k2, n2);
                x[e] = ex2_approx(y.x);
                x[e + 1] = ex2_approx(y.y);
              }
              if (static_cast<unsigned>(target - col0) < 32u) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (target - col0 == e) x[e] -= 1.f;
              }
              if (col0 + 32 > p.V) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (col0 + e >= p.V) x[e] = 0.f;
              }
              const float2 d2 = make_float2(dloss, dloss);
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                const float2 y = fmul2(make_float2(x[e], x[e + 1]), d2);
                x[e] = y.x;
                x[e + 1] = y.y;
              }
            }
            if (kMode == kDw && work.k == 0) {  // no scored row: nothing was multiplied
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = 0.f;
            }
            // 128 bytes of a row a buffer: 32 columns of fp32, 64 of bf16 (two chunks).
            const bool opens = kMode == kDh || (c & 1) == 0, closes = kMode == kDh || (c & 1) == 1;
            uint8_t* buf = sm.out[qw][chunk & 1];
            if (opens) {
              if (lane == 0) bulk_wait_read<1>();  // the store before the last has left this buffer
              __syncwarp();
            }
            uint8_t* dst = buf + lane * 128;
            if (kMode == kDh) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                *reinterpret_cast<float4*>(dst + ((e ^ (lane & 7)) << 4)) =
                    make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                *reinterpret_cast<uint4*>(dst + (((4 * (c & 1) + e) ^ (lane & 7)) << 4)) =
                    make_uint4(pack_bf16x2(x[8 * e], x[8 * e + 1]), pack_bf16x2(x[8 * e + 2], x[8 * e + 3]),
                               pack_bf16x2(x[8 * e + 4], x[8 * e + 5]), pack_bf16x2(x[8 * e + 6], x[8 * e + 7]));
            }
            if (closes) {
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) {
                const int r0 = tl.m * kBM + qw * 32;
                if (kMode == kGrad) tma_store_2d(&mo, buf, tl.n * p.bn + 32 * (c - 1), r0);
                if (kMode == kDw) {
                  const int col = tl.n * p.bn + 32 * (c - 1);
                  if (p.v0 + r0 < p.rows_out && col < p.cols_out) tma_store_2d(&mo, buf, col, p.v0 + r0);
                }
                if (kMode == kDh) {
                  const int y = tl.split * work.row_blocks * kBM + r0, col = tl.n * p.bn + 32 * c;
                  if (col < p.cols_out) {
                    if (!p.add)
                      tma_store_2d(&mo, buf, col, y);
                    else if (tl.k1 > tl.k0)
                      tma_add_2d(&mo, buf, col, y);
                  }
                }
                bulk_commit();
              }
              ++chunk;
            }
          }
        }
        s += ts;
      }
      if (!ok) break;
      if (kMode == kStats)
        p.part[static_cast<int64_t>(item) * kBM + t_row] = make_float2(m, s);
    }
    if (kMode != kStats && lane == 0) bulk_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------- scored rows

struct GatherParams {
  const int* target;
  const void* hidden;   // bf16, any alignment
  const float* lse;     // gradients only
  const float* dloss;
  int64_t s_hidden;
  int N, V, d, d_pad, rows_per_cta;
  Plan* plan;
  int* place;           // [N] place of a row among the scored ones, -1: not scored
  int* to_target;
  float* to_lse2;
  float* to_dloss;
  uint4* to_hidden;     // [., d_pad]
  float* loss;          // loss only: 0 for rows that are not scored
  float* lse_out;
  int tiles, kblocks, ctas, max_rows;  // gradients: what the K splits of dh depend on
};

constexpr int kGatherThreads = 256;

// The K splits of dh that leave the busiest CTA the fewest steps: a tile also costs
// about 16 steps (of 64, 128 x 256: 0.34 us) for writing and reading its fp32 sums. A
// lane of a warp looks at two numbers of splits (one thread at all of them: 8 us).
__device__ int choose_splits(const GatherParams& p, int n) {
  const int lane = threadIdx.x & 31, blocks = (n + kBM - 1) / kBM;
  unsigned best = 0xFFFFFFFFu;
  int splits = 1;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = lane + 32 * k + 1;
    const bool fits = s == 1 || (s <= p.kblocks && blocks <= p.max_rows / kBM / s);
    const unsigned rounds = (static_cast<unsigned>(blocks) * p.tiles * s + p.ctas - 1) / p.ctas;
    const unsigned cost = fits ? rounds * ((p.kblocks + s - 1) / s + 16) : 0xFFFFFFFFu;
    if (cost < best) {
      best = cost;
      splits = s;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned c = __shfl_xor_sync(0xffffffffu, best, o);
    const int s = __shfl_xor_sync(0xffffffffu, splits, o);
    if (c < best || (c == best && s < splits)) {
      best = c;
      splits = s;
    }
  }
  return splits;
}

__device__ int block_count(int v, int* sums) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int i = 0; i < kGatherThreads / 32; ++i) v += sums[i];
  return v;
}

// Each CTA counts the scored rows before its own and copies its own behind them; the
// last one knows their number and fills the last block of 128 rows with zeros.
__global__ void __launch_bounds__(kGatherThreads) loss_gather_kernel(const GatherParams p) {
  __shared__ int sums[kGatherThreads / 32];
  __shared__ int source[kGatherThreads];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  wait_for_previous();
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * p.rows_per_cta;
  const int64_t r1 = r0 + p.rows_per_cta < p.N ? r0 + p.rows_per_cta : p.N;
  const auto scored = [&](int t) { return static_cast<unsigned>(t) < static_cast<unsigned>(p.V); };
  int before = 0;
#pragma unroll 8
  for (int64_t r = threadIdx.x; r < r0; r += kGatherThreads) before += scored(p.target[r]);
  before = block_count(before, sums);
  const int vecs = p.d_pad / 8, full = p.d / 8;
  const bool aligned = ((reinterpret_cast<uintptr_t>(p.hidden) | static_cast<uintptr_t>(p.s_hidden * 2)) & 15) == 0;
  for (int64_t base = r0; base < r1; base += kGatherThreads) {
    const int64_t r = base + threadIdx.x;
    const int t = r < r1 ? p.target[r] : -1;
    const bool on = scored(t);
    const unsigned vote = __ballot_sync(0xffffffffu, on);
    __syncthreads();  // sums and source of the round before have been read
    if (lane == 0) sums[warp] = __popc(vote);
    __syncthreads();
    int at = __popc(vote & ((1u << lane) - 1)), total = 0;
#pragma unroll
    for (int i = 0; i < kGatherThreads / 32; ++i) {
      if (i < warp) at += sums[i];
      total += sums[i];
    }
    if (on) {
      source[at] = static_cast<int>(r - base);
      p.to_target[before + at] = t;
      if (p.to_lse2) {
        p.to_lse2[before + at] = p.lse[r] * kLog2e;
        p.to_dloss[before + at] = p.dloss[r];
      }
    }
    if (r < r1) {
      p.place[r] = on ? before + at : -1;
      if (!on && p.loss) {
        p.loss[r] = 0.f;
        p.lse_out[r] = 0.f;
      }
    }
    __syncthreads();
    for (int k = warp; k < total; k += kGatherThreads / 32) {
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.hidden) + (base + source[k]) * p.s_hidden;
      uint4* dst = p.to_hidden + static_cast<int64_t>(before + k) * vecs;
#pragma unroll 4
      for (int i = lane; i < vecs; i += 32) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (i < full) {
          if (aligned) {
            v = reinterpret_cast<const uint4*>(src)[i];
          } else {
            const unsigned short* e = reinterpret_cast<const unsigned short*>(src) + 8 * i;
            v = make_uint4(e[0] | static_cast<uint32_t>(e[1]) << 16, e[2] | static_cast<uint32_t>(e[3]) << 16,
                           e[4] | static_cast<uint32_t>(e[5]) << 16, e[6] | static_cast<uint32_t>(e[7]) << 16);
          }
        }
        dst[i] = v;
      }
    }
    before += total;
  }
  if (blockIdx.x != gridDim.x - 1) return;
  const int n = before, end = (n + kBM - 1) / kBM * kBM;
  if (warp == 0) {
    const int splits = p.tiles ? choose_splits(p, n) : 1;
    if (lane == 0) {
      p.plan->n = n;
      p.plan->splits = splits;
    }
  }
  for (int r = n + threadIdx.x; r < end; r += kGatherThreads) {
    p.to_target[r] = -1;
    if (p.to_lse2) p.to_lse2[r] = p.to_dloss[r] = 0.f;
  }
  for (int64_t i = static_cast<int64_t>(n) * vecs + threadIdx.x; i < static_cast<int64_t>(end) * vecs; i += kGatherThreads)
    p.to_hidden[i] = make_uint4(0, 0, 0, 0);
}

// ---------------------------------------------------------------- results

// Joins the parts of each scored row, a warp a row.
constexpr int kCombineThreads = 256;
__global__ void __launch_bounds__(kCombineThreads)
    loss_combine_kernel(const Plan* plan, const int* place, const float2* part, const float* x_target, int N, int parts,
                        float* loss, float* lse) {
  wait_for_previous();
  const int64_t r = (static_cast<int64_t>(blockIdx.x) * kCombineThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (r >= N) return;
  const int c = place[r];
  if (c < 0) return;  // written by the first launch
  const int64_t step = static_cast<int64_t>((plan->n + kBM - 1) / kBM) * kBM;
  constexpr int kPer = (kLossMaxParts + 31) / 32;
  float2 v[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) v[j] = lane + 32 * j < parts ? part[(lane + 32 * j) * step + c] : make_float2(-INFINITY, 0.f);
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < kPer; ++j) m = fmaxf(m, v[j].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < kPer; ++j) s += v[j].x == -INFINITY ? v[j].y : v[j].y * expf(v[j].x - m);  // 0 or a NaN without a maximum
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) {
    const float ln = m == -INFINITY ? NAN : logf(s);  // every logit -inf or NaN: no distribution
    lse[r] = m + ln;
    loss[r] = (m - x_target[c]) + ln;
  }
}

// d_hidden: the splits' sums of each scored row, zeros for the others; four columns a
// thread, eight splits' loads in flight.
constexpr int kFinishThreads = 128;
__global__ void __launch_bounds__(kFinishThreads)
    loss_dhidden_kernel(const Plan* plan, const int* place, const float* part, int N, int d, int d_pad, __nv_bfloat16* out,
                        int64_t s_out, int aligned) {
  wait_for_previous();
  const int vecs = d / 4, splits = plan->splits;
  const int64_t step = static_cast<int64_t>((plan->n + kBM - 1) / kBM) * kBM * d_pad;
  const int64_t total = static_cast<int64_t>(N) * vecs;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kFinishThreads + threadIdx.x; i < total;
       i += static_cast<int64_t>(gridDim.x) * kFinishThreads) {
    const int64_t r = i / vecs;
    const int col = static_cast<int>(i - r * vecs) * 4, c = place[r];
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c >= 0) {
      const float* src = part + static_cast<int64_t>(c) * d_pad + col;
      for (int s = 0; s < splits; s += 8) {
        float4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          v[k] = s + k < splits ? *reinterpret_cast<const float4*>(src + (s + k) * step) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) a = make_float4(a.x + v[k].x, a.y + v[k].y, a.z + v[k].z, a.w + v[k].w);
      }
    }
    const uint2 o = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
    __nv_bfloat16* dst = out + r * s_out + col;
    if (aligned) {
      *reinterpret_cast<uint2*>(dst) = o;
    } else {
      unsigned short* e = reinterpret_cast<unsigned short*>(dst);
      e[0] = static_cast<unsigned short>(o.x & 0xFFFFu);
      e[1] = static_cast<unsigned short>(o.x >> 16);
      e[2] = static_cast<unsigned short>(o.y & 0xFFFFu);
      e[3] = static_cast<unsigned short>(o.y >> 16);
    }
  }
}

// ---------------------------------------------------------------- host side

int sm_count() {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

// Columns of a tile: 256, or 128 or 64 where 256 leave SMs without a tile or much of the
// last tile empty (narrow tiles read their other operand more often: a column counts
// 1.12 and 1.36 times, as in the projection's own choice). With one CTA: by the last
// tile alone (dw has tiles enough, dh is split).
int choose_bn(int64_t cols, int64_t row_tiles, int ctas) {
  int best = 256;
  double best_cost = 1e300;
  for (int bn = 256; bn >= 64; bn /= 2) {
    const int64_t tiles = (cols + bn - 1) / bn * row_tiles, rounds = (tiles + ctas - 1) / ctas;
    const double cost = static_cast<double>(rounds) * (bn / 256.0 * 0.88 + 0.12);
    if (cost < best_cost - 1e-9) {
      best_cost = cost;
      best = bn;
    }
  }
  return best;
}

template <int kMode>
int launch_product(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mo, const Params& p, int64_t items, int sms,
                   cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(loss_product_kernel<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(kSmemBytes));
  const int64_t grid = items < sms ? items : sms;
  if (e == cudaSuccess)
    e = launch_overlapped(loss_product_kernel<kMode>, dim3(static_cast<unsigned>(grid)), kThreads, kSmemBytes, stream, 1, true, ma,
                          mb, mo, p);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "projection loss launch: %s", cudaGetErrorString(e));
}

// Places of the workspace, from its start.
struct Layout {
  int64_t n_pad, d_pad;
  size_t plan, place, target, lse2, dloss, hidden, x_target, part, sums, g;  // byte offsets
  size_t sums_rows;  // gradients: rows of fp32 sums
};

size_t take(size_t* at, size_t bytes) {
  const size_t here = *at;
  *at += (bytes + 255) / 256 * 256;
  return here;
}

Layout layout_of(int64_t N, int64_t d, bool grad) {
  Layout l = {};
  l.n_pad = (N + kBM - 1) / kBM * kBM;
  l.d_pad = (d + kBK - 1) / kBK * kBK;
  size_t at = 0;
  l.plan = take(&at, sizeof(Plan));
  l.place = take(&at, N * 4);
  l.target = take(&at, l.n_pad * 4);
  l.hidden = take(&at, l.n_pad * l.d_pad * 2);
  if (!grad) {
    l.x_target = take(&at, l.n_pad * 4);
    l.part = take(&at, static_cast<size_t>(kLossMaxParts) * l.n_pad * 8);
  } else {
    l.lse2 = take(&at, l.n_pad * 4);
    l.dloss = take(&at, l.n_pad * 4);
    // Room for splits of dh: up to 32 of them, 192 MB, and one in any case.
    const int64_t most = (int64_t{192} << 20) / (l.d_pad * 4) / kBM * kBM;
    int64_t rows = 32 * l.n_pad < most ? 32 * l.n_pad : most;
    if (rows < l.n_pad) rows = l.n_pad;
    l.sums_rows = static_cast<size_t>(rows);
    l.sums = take(&at, l.sums_rows * l.d_pad * 4);
  }
  l.g = at;
  return l;
}

int launch_gather(const LossArgs& a, const Layout& l, GatherParams g, cudaStream_t stream) {
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  g.target = a.targets;
  g.hidden = a.hidden;
  g.s_hidden = a.s_hidden;
  g.N = static_cast<int>(a.N);
  g.V = static_cast<int>(a.V);
  g.d = static_cast<int>(a.d);
  g.d_pad = static_cast<int>(l.d_pad);
  g.plan = reinterpret_cast<Plan*>(ws + l.plan);
  g.place = reinterpret_cast<int*>(ws + l.place);
  g.to_target = reinterpret_cast<int*>(ws + l.target);
  g.to_hidden = reinterpret_cast<uint4*>(ws + l.hidden);
  // 16 rows a CTA, more where every CTA would otherwise count very many rows before its own.
  int64_t rows = 16;
  while (rows < kGatherThreads && a.N > rows * 2048) rows *= 2;
  g.rows_per_cta = static_cast<int>(rows);
  const cudaError_t e = launch_overlapped(loss_gather_kernel, dim3(static_cast<unsigned>((a.N + rows - 1) / rows)), kGatherThreads, 0,
                                          stream, 1, true, g);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "scored rows launch: %s", cudaGetErrorString(e));
}

Params common_params(const LossArgs& a, const Layout& l) {
  Params p = {};
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  p.plan = reinterpret_cast<Plan*>(ws + l.plan);
  p.V = static_cast<int>(a.V);
  p.target = reinterpret_cast<int*>(ws + l.target);
  p.err = device_error_word();
  p.wait_ns = wait_budget_ns();
  return p;
}

}  // namespace

size_t loss_workspace_bytes(int64_t N, int64_t d) { return layout_of(N, d, false).g; }

size_t loss_grad_workspace_bytes(int64_t N, int64_t V, int64_t d, int64_t piece) {
  const Layout l = layout_of(N, d, true);
  const int64_t all = (V + 255) / 256 * 256;
  // 2 GB of g unless told otherwise, but not under 1024 columns: the fewer pieces, the fewer tails.
  int64_t cols = piece > 0 ? (piece + 255) / 256 * 256 : (int64_t{1} << 31) / (l.n_pad * 2) / 256 * 256;
  if (piece <= 0 && cols < 1024) cols = 1024;
  if (cols > all) cols = all;
  return l.g + static_cast<size_t>(l.n_pad) * cols * 2;
}

int launch_loss(const LossArgs& a, cudaStream_t stream) {
  const Layout l = layout_of(a.N, a.d, false);
  const int sms = sm_count();
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  GatherParams g = {};
  g.loss = a.loss;
  g.lse_out = a.lse_out;
  int st;
  if ((st = launch_gather(a, l, g, stream)) != DLM_OK) return st;
  Params p = common_params(a, l);
  const int64_t row_blocks = l.n_pad / kBM;
  p.kblocks = static_cast<int>(l.d_pad / kBK);
  p.bn = choose_bn(a.V, row_blocks, sms);
  p.tiles = static_cast<int>((a.V + p.bn - 1) / p.bn);
  p.parts = p.tiles < kLossMaxParts ? p.tiles : kLossMaxParts;
  p.a_rows = a.N < kBM ? static_cast<int>((a.N + 7) / 8 * 8) : kBM;
  p.part = reinterpret_cast<float2*>(ws + l.part);
  p.x_target = reinterpret_cast<float*>(ws + l.x_target);
  CUtensorMap mh, mw;
  if ((st = make_matrix_map(&mh, ws + l.hidden, true, l.n_pad, l.d_pad, l.d_pad, p.a_rows)) != DLM_OK) return st;
  if ((st = make_matrix_map(&mw, a.weight, true, a.V, a.d, a.s_weight, p.bn)) != DLM_OK) return st;
  if ((st = launch_product<kStats>(mh, mw, mw, p, p.parts * row_blocks, sms, stream)) != DLM_OK) return st;
  const cudaError_t e = launch_overlapped(
      loss_combine_kernel, dim3(static_cast<unsigned>((a.N * 32 + kCombineThreads - 1) / kCombineThreads)), kCombineThreads, 0, stream,
      1, true, p.plan, reinterpret_cast<const int*>(ws + l.place), static_cast<const float2*>(p.part),
      static_cast<const float*>(p.x_target), static_cast<int>(a.N), p.parts, a.loss, a.lse_out);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "loss combine launch: %s", cudaGetErrorString(e));
}

int launch_loss_grad(const LossArgs& a, cudaStream_t stream) {
  const Layout l = layout_of(a.N, a.d, true);
  const int sms = sm_count();
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  const int64_t all = (a.V + 255) / 256 * 256;
  int64_t cols = static_cast<int64_t>((a.workspace_bytes - l.g) / (static_cast<size_t>(l.n_pad) * 2)) / 256 * 256;
  if (cols > all) cols = all;
  const int64_t row_blocks = l.n_pad / kBM;
  const int bn_d = choose_bn(a.d, 1, 1);

  GatherParams g = {};
  g.lse = a.lse;
  g.dloss = a.dloss;
  g.to_lse2 = reinterpret_cast<float*>(ws + l.lse2);
  g.to_dloss = reinterpret_cast<float*>(ws + l.dloss);
  g.tiles = static_cast<int>((a.d + bn_d - 1) / bn_d);
  g.kblocks = static_cast<int>(((cols < a.V ? cols : a.V) + kBK - 1) / kBK);
  g.ctas = sms;
  g.max_rows = l.sums_rows > 0x7FFFFFFF ? 0x7FFFFFFF : static_cast<int>(l.sums_rows);
  int st;
  if ((st = launch_gather(a, l, g, stream)) != DLM_OK) return st;

  CUtensorMap h_k, h_mn, w_k, w_mn, g_k, g_mn, g_out, dw_out, dh_out;
  const Params base = common_params(a, l);
  const int bn_v = choose_bn(a.V < cols ? a.V : cols, row_blocks, sms);
  if ((st = make_matrix_map(&h_k, ws + l.hidden, true, l.n_pad, l.d_pad, l.d_pad, kBM)) != DLM_OK) return st;
  if ((st = make_matrix_map(&h_mn, ws + l.hidden, true, l.n_pad, l.d_pad, l.d_pad, 64)) != DLM_OK) return st;
  if ((st = make_matrix_map(&w_k, a.weight, true, a.V, a.d, a.s_weight, bn_v)) != DLM_OK) return st;
  if ((st = make_matrix_map(&w_mn, a.weight, true, a.V, a.d, a.s_weight, 64)) != DLM_OK) return st;
  if ((st = make_matrix_map(&g_k, ws + l.g, true, l.n_pad, cols, cols, kBM)) != DLM_OK) return st;
  if ((st = make_matrix_map(&g_mn, ws + l.g, true, l.n_pad, cols, cols, 64)) != DLM_OK) return st;
  if ((st = make_matrix_map(&g_out, ws + l.g, true, l.n_pad, cols, cols, 32)) != DLM_OK) return st;
  if (a.d_weight && (st = make_matrix_map(&dw_out, a.d_weight, true, a.V, a.d, a.s_dweight, 32)) != DLM_OK) return st;
  if ((st = make_matrix_map(&dh_out, ws + l.sums, false, static_cast<int64_t>(l.sums_rows), l.d_pad, l.d_pad, 32)) != DLM_OK) return st;

  for (int64_t v0 = 0; v0 < a.V; v0 += cols) {
    const int64_t vc = a.V - v0 < cols ? a.V - v0 : cols;
    Params p = base;
    p.v0 = static_cast<int>(v0);
    p.kblocks = static_cast<int>(l.d_pad / kBK);
    p.bn = bn_v;
    p.tiles = static_cast<int>((vc + bn_v - 1) / bn_v);
    p.lse2 = g.to_lse2;
    p.dloss = g.to_dloss;
    if ((st = launch_product<kGrad>(h_k, w_k, g_out, p, p.tiles * row_blocks, sms, stream)) != DLM_OK) return st;
    p.bn = bn_d;
    p.tiles = g.tiles;
    if (a.d_weight) {
      p.rows_out = p.V;
      p.cols_out = static_cast<int>(a.d);
      p.parts = static_cast<int>((vc + kBM - 1) / kBM);
      if ((st = launch_product<kDw>(g_mn, h_mn, dw_out, p, static_cast<int64_t>(p.parts) * p.tiles, sms, stream)) != DLM_OK) return st;
    }
    if (a.d_hidden) {
      p.kblocks = static_cast<int>((vc + kBK - 1) / kBK);
      p.add = v0 > 0;
      p.cols_out = static_cast<int>(l.d_pad);
      if ((st = launch_product<kDh>(g_k, w_mn, dh_out, p, sms, sms, stream)) != DLM_OK) return st;
    }
  }
  if (!a.d_hidden) return DLM_OK;
  const int64_t vecs = a.N * (a.d / 4);
  const int64_t want = (vecs + kFinishThreads - 1) / kFinishThreads, most = static_cast<int64_t>(sms) * 16;
  const bool aligned = ((reinterpret_cast<uintptr_t>(a.d_hidden) | static_cast<uintptr_t>(a.s_dhidden * 2)) & 7) == 0;
  const cudaError_t e = launch_overlapped(
      loss_dhidden_kernel, dim3(static_cast<unsigned>(want < most ? want : most)), kFinishThreads, 0, stream, 1, true, base.plan,
      reinterpret_cast<const int*>(ws + l.place), reinterpret_cast<const float*>(ws + l.sums), static_cast<int>(a.N),
      static_cast<int>(a.d), static_cast<int>(l.d_pad), static_cast<__nv_bfloat16*>(a.d_hidden), a.s_dhidden, aligned ? 1 : 0);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "hidden gradient launch: %s", cudaGetErrorString(e));
}

}  // namespace dlm
