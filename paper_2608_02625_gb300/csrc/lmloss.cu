// Cross entropy of given tokens under the output projection, and its gradients, on
// the tensor cores; the N x V logits are never stored.
//
//   x[r, v] = hidden[r] . weight[v],  lse[r] = ln sum_v e^x,  loss[r] = lse[r] - x[r, t_r]
//   g[r, v] = dloss[r] (e^(x - lse[r]) - [v = t_r])
//   d_hidden = g weight,   d_weight = g^T hidden
//
// Rows without a target (outside [0, V)) are not scored: the first launch copies the
// hidden states of the others, in their order, to the workspace (n rows), so the products
// take time for scored rows alone -- of a masked diffusion batch a quarter, say -- and
// their number stays on the GPU.
//
// The products run through one persistent kernel in three modes, 128 x bn output tiles a
// CTA (bn up to 256), K steps of 64 through a ring of 192 KB:
//   stats  x = H W^T     per row and part of the vocabulary: maximum, sum of e^(x - m),
//                        and the target's logit; loss_combine_kernel joins the parts
//   grad   x = H W^T     g of one piece of the vocabulary, rounded to bf16, to the workspace
//   back   g^T H         dw: a piece of d_weight, bf16, and
//          g W           dh: fp32 sums over the piece, added to those of the pieces before
//                        it; split over K where there are too few tiles for every SM
// With many rows two CTAs share a tile of 256 rows (cta_group::2): each loads half of B,
// which an MMA of one CTA's reads whole, and shared memory feeds the MMAs with fewer
// pauses (4096 x 20000 x 2048: grad 203 -> 175 us, 90 % of the tensor pipe's cycles; dw
// 247 -> 207, dh 250 -> 207). What such an MMA reads most of, B, is K-major (with an
// MN-major B both products keep the pipe 73 % busy): dw multiplies g^T by the hidden states
// transposed once, dh is computed transposed, W^T g^T, and turned back with its rounding.
// Single CTAs, with few rows or little width, take the operands as they lie.
// g is rounded to bf16 because the tensor cores take it so: every term of d_hidden and
// d_weight is off by at most 2^-8 relative, as the result is by its own rounding to bf16;
// all sums are fp32. The one large term, the target's, would stand out: of d_hidden its
// rounding is made good at the end, with the target's row of the weight, and where every
// row has the same dloss, the mean's, g is rounded without dloss's mantissa, which leaves
// -(1 - p) nearly exact. Warp 0 loads by TMA, warp 1 issues tcgen05.mma (both operands in
// shared memory), warps 4-11 read the fp32 accumulators (two, so a tile's epilogue runs
// under the next one's K loop) and write their tiles through shared memory by TMA.
// Every wait is bounded; on expiry the kernel sets DLM_DEVERR_TIMEOUT, lets what it has on
// its way land (a pair: in both CTAs) and exits.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"
#include "dlm_tmap.h"

namespace cg = cooperative_groups;

namespace dlm {
namespace {

constexpr int kBM = 128;          // a CTA's rows of an output tile = TMEM lanes
constexpr int kBK = 64;           // K of a stage: 128 bytes of bf16
constexpr int kMaxBN = 256;
constexpr int kThreads = 384;     // warp 0 TMA, warp 1 MMA, warps 4-11 epilogue
constexpr int kEpiWarp0 = 4, kEpiWarps = 8;
constexpr int kABytes = kBM * kBK * 2;
constexpr int kBoxBytes = 64 * 128;          // an MN-major box: 64 K rows of 64 columns
constexpr uint32_t kTmemCols = 2 * kMaxBN;   // two accumulators
constexpr float kLog2e = 1.4426950408889634f;
// Which calls may run in pairs of CTAs, by rows and width, and whether they do, by the number
// of scored rows, which the GPU alone knows: both forms are launched, and one of them ends at
// once (a gradient of 640 rows 893 -> 916 us, of 4096 no more; a quarter of 512 rows 513 ->
// 328, of 1024 567 -> 467). V = 151552, d = 2048, graph us, single and pairs: loss 129 rows 134,
// 121; 256 137, 127; 320 (of the pair's two tiles one is nearly empty) 184, 200; 448 232, 217;
// gradients 256 460, 559; 320 601, 619; 448 771, 668; 512 712, 684. By width: loss 4096 x 1024
// 778, 741; x 512 400, 419 (the epilogues of both wait for the slower); gradients 4096 x 512
// 1452, 1300; x 256 857, 803; x 64 661, 718; 2048 x 256 (V = 20000) 82, 83. Of small products
// pairs make too few tiles, each later done: gradients of 500 x 4000 x 512 31, 57;
// 700 x 10000 x 1024 59, 65; 1024 x 10000 x 1024 80, 79; 1024 x 20000 x 1024 120, 109; loss
// 1024 x 4000 x 2048 27, 29; 2048 x 4000 x 2048 41, 41; 1024 x 10000 x 2048 61, 60.
constexpr double kPairLoss = 16e9, kPairGradients = 10e9;  // n V d
bool pairs_have_room(int64_t N, int64_t d) { return N > 3 * kBM && d >= (N >= 4096 ? 256 : 512); }  // gradients' workspace
// The scored rows from which pairs pay for themselves; 0: never, in a call of N rows.
int pair_rows(int64_t N, int64_t V, int64_t d, bool gradients) {
  if (gradients ? !pairs_have_room(N, d) : N <= kBM || d < 1024) return 0;
  const double rows = ceil((gradients ? kPairGradients : kPairLoss) / (static_cast<double>(V) * static_cast<double>(d)));
  return rows > static_cast<double>(N) ? 0 : rows < 1.0 ? 1 : static_cast<int>(rows);
}
__device__ bool pairs_pay(int n, int from, bool gradients) {
  return n >= from && (n > 3 * kBM || (!gradients && n > kBM && n <= 2 * kBM));
}

enum Mode { kStats, kGrad, kBack };

// kCtas: CTAs that share a tile, 1 or 2 (a pair holds half of B each).
template <int kCtas>
struct Smem {
  static constexpr int kStages = kCtas == 2 ? 6 : 4;  // 192 KB
  static constexpr int kBBytes = kMaxBN / kCtas * kBK * 2;
  alignas(1024) uint8_t a[kStages][kABytes];
  alignas(1024) uint8_t b[kStages][kBBytes];
  alignas(1024) uint8_t out[kEpiWarps][32 * 128];  // per epilogue warp, 32 rows x 128 bytes
  uint64_t full[kStages];   // stage loaded            (TMA -> MMA; a pair's: in the leader)
  uint64_t empty[kStages];  // stage read by its MMAs  (MMA -> TMA)
  uint64_t acc_full[2];     // accumulator complete    (MMA -> epilogue)
  uint64_t acc_empty[2];    // accumulator read out    (epilogue -> MMA; a pair's: in the leader)
  uint64_t done;            // every MMA completed     (teardown; a pair's: in the leader)
  uint32_t tmem_base;
  int abort;
  // Of a pair, in both CTAs: what each has loaded, what the leader's MMAs have committed, and
  // whether a role of either has given up.
  int loads[2], mma_steps, mma_tiles, gave_up;
};
template <int kCtas>
constexpr size_t smem_bytes() {
  return sizeof(Smem<kCtas>) + 1024;
}
static_assert(smem_bytes<1>() <= 227 * 1024 && smem_bytes<2>() <= 227 * 1024, "shared memory of a CTA");

// What the first launch leaves for the others.
struct Plan {
  int n;        // scored rows
  int pairs;    // whether CTAs work in pairs
  int splits;   // K splits of dh
  float scale;  // what g is divided by: the first scored row's dloss, its power of two taken out
};

struct Params {
  const Plan* plan;
  int either;           // both forms are launched: this one works if the plan says so
  int V;
  int kblocks;          // stats, grad: K steps (of d);  back: those of dh (of the piece)
  int bn;               // columns of a tile
  int tiles;            // stats, grad: vocabulary tiles;  back: dw's tiles of d
  int dh_tiles;         // back: dh's tiles of d
  int parts;            // stats: parts of the vocabulary;  back: dw's tiles of the piece's rows
  int v0;               // first vocabulary column of the piece
  int n_pad;            // rows of a panel of g
  int a_rows;           // stats: rows of the hidden box
  int want_dw, want_dh;
  int add;              // dh: add to what the pieces before left
  int dw_rows, dw_cols, dh_cols;  // extents of what is written (dh_cols: single CTAs)
  const int* target;    // of each scored row
  const float* lse2;    // lse log2(e)
  const float* dloss;
  float* rest;          // grad: what the rounding of g took from the target's, of each scored row
  float2* part;         // stats: (maximum, sum) [half of the warps][part][row]
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

// *v = x where i == e. (Selects in C++ become an index into an array in local memory.)
__device__ __forceinline__ void take_if(int i, int e, float x, float* v) {
  asm("{\n.reg .pred q;\nsetp.eq.s32 q, %1, %2;\nselp.f32 %0, %3, %0, q;\n}" : "+f"(*v) : "r"(i), "r"(e), "f"(x));
}

// One output tile and its K steps [k0, k1). m, n: its row and column tiles; dw: of
// d_weight (else, in back, of d_hidden).
struct Tile {
  int m, n, k0, k1, split;
  bool dw;
};

// What tiles cost, in K steps fed from L2 (of 64; 0.27 to 0.34 us). A step of dh waits for
// HBM where few row blocks share the weight that it reads; its tile is written and read
// as fp32 sums. dw's takes no less than writing it.
__device__ __forceinline__ float dh_cost(int steps, int row_blocks) { return steps * fmaxf(1.f, 2.f / row_blocks) + 16.f; }
__device__ __forceinline__ float dw_cost(int steps) { return max(steps, 4) + 1.f; }

// The work of a launch: items, each a run of tiles [t0, t1) (one tile but for stats).
//
// back: every worker takes tiles of dh, one round of all workers after another; those
// without one in the last round turn to dw meanwhile, the others when they are done. The
// rounds of each phase keep the workers on neighbouring tiles, which share their operands
// in L2. (dw and dh in launches of their own leave workers without a tile in both last
// rounds: 4096 x 65536 x 2048 dh 85 % of the SM cycles used.)
template <int kMode, int kCtas>
struct Work {
  static constexpr int kRows = kBM * kCtas;  // rows of a tile
  // Columns of a tile: a pair's of dh are rows of g, 256 of them.
  static __device__ __forceinline__ int bn(const Params& p, const Tile& t) {
    return kMode == kBack && kCtas == 2 && !t.dw ? kMaxBN : p.bn;
  }
  int items, row_blocks, k, splits;
  int k_dw, k_tail;               // back: dw's K steps, and the 16s of the last
  int dh, dw, left, meanwhile;    // back: tiles of each, dh's in its last round, dw's a worker meanwhile

  __device__ Work(const Params& p, int workers) {
    const int n = p.plan->n;
    row_blocks = (n + kRows - 1) / kRows;
    splits = p.plan->splits;
    k = p.kblocks;
    items = kMode == kStats ? p.parts * row_blocks : p.tiles * row_blocks;
    if (kMode != kBack) return;
    k_dw = (n + kBK - 1) / kBK;
    k_tail = (n - (k_dw - 1) * kBK + 15) / 16;
    dh = p.want_dh ? splits * row_blocks * p.dh_tiles : 0;
    dw = p.want_dw ? p.parts * p.tiles : 0;
    left = dh % workers;
    meanwhile = left ? static_cast<int>(dh_cost(k / splits, row_blocks) / dw_cost(k_dw)) : 0;
  }
  // The worker's j-th item, -1: none.
  __device__ __forceinline__ int item(int worker, int workers, int j) const {
    if (kMode != kBack) {
      const int i = worker + j * workers;
      return i < items ? i : -1;
    }
    const int own = dh / workers + (worker < left ? 1 : 0);
    if (j < own) return j * workers + worker;
    j -= own;
    int t;
    if (left && worker >= left && j < meanwhile) {
      t = j * (workers - left) + worker - left;
    } else {
      if (left && worker >= left) j -= meanwhile;
      t = meanwhile * (workers - left) + j * workers + worker;
    }
    return t < dw ? dh + t : -1;
  }
  __device__ __forceinline__ int first(const Params& p, int item) const {
    return kMode == kStats ? static_cast<int>(static_cast<long long>(p.tiles) * (item / row_blocks) / p.parts) : 0;
  }
  __device__ __forceinline__ int last(const Params& p, int item) const {
    return kMode == kStats ? static_cast<int>(static_cast<long long>(p.tiles) * (item / row_blocks + 1) / p.parts) : 1;
  }
  // Items that run at the same time share vocabulary tiles (stats, grad: the row block
  // changes first) or the rows of g (back: the tile of d changes first).
  __device__ __forceinline__ Tile tile(const Params& p, int item, int t) const {
    if (kMode == kStats) return {item % row_blocks, t, 0, k, 0, false};
    if (kMode == kGrad) return {item % row_blocks, item / row_blocks, 0, k, 0, false};
    if (item >= dh) return {(item - dh) / p.tiles, (item - dh) % p.tiles, 0, k_dw, 0, true};
    const int per = row_blocks * p.dh_tiles, split = item / per, rest = item % per;
    const int rows = rest / p.dh_tiles, cols = rest % p.dh_tiles;
    return {kCtas == 2 ? cols : rows, kCtas == 2 ? rows : cols, static_cast<int>(static_cast<long long>(k) * split / splits),
            static_cast<int>(static_cast<long long>(k) * (split + 1) / splits), split, false};
  }
};

// ma, mb: the operands' maps; mo: the map written (none for stats). back: those of dh, and
// mda, mdb, mdo of dw.
template <int kMode, int kCtas>
__global__ void __launch_bounds__(kThreads, 1)
    loss_product_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
                        const __grid_constant__ CUtensorMap mo, const __grid_constant__ CUtensorMap mda,
                        const __grid_constant__ CUtensorMap mdb, const __grid_constant__ CUtensorMap mdo, const Params p) {
  using Sm = Smem<kCtas>;
  constexpr int kStages = Sm::kStages, kBBytes = Sm::kBBytes, kRows = kBM * kCtas;
  extern __shared__ uint8_t smem_raw[];
  Sm& sm = *reinterpret_cast<Sm*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int rank = kCtas == 2 ? static_cast<int>(blockIdx.x & 1) : 0;  // in the pair
  const int worker = static_cast<int>(blockIdx.x) / kCtas, workers = static_cast<int>(gridDim.x) / kCtas;

  if (p.either) {
    wait_for_previous();
    if (p.plan->pairs != (kCtas == 2)) return;
  }
  if (threadIdx.x == 32 * kEpiWarp0) {  // parameters, not memory that another kernel writes
    prefetch_tmap(&ma);
    prefetch_tmap(&mb);
    if (kMode == kGrad || (kMode == kBack && p.want_dh)) prefetch_tmap(&mo);
    if (kMode == kBack && p.want_dw) {
      prefetch_tmap(&mda);
      prefetch_tmap(&mdb);
      prefetch_tmap(&mdo);
    }
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.acc_full[i], 1);
      mbar_init(&sm.acc_empty[i], kEpiWarps * kCtas);
    }
    mbar_init(&sm.done, 1);
    sm.abort = 0;
    sm.gave_up = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    if (kCtas == 2) {
      tmem_alloc_pair(&sm.tmem_base, kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(&sm.tmem_base, kTmemCols);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  if (kCtas == 2)
    cg::this_cluster().sync();  // the other CTA's barriers and tensor memory are there too
  else
    __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  volatile int* abort = &sm.abort;
  wait_for_previous();
  const Work<kMode, kCtas> work(p, workers);
  // A role of a pair that ends early (a whole warp): see the end.
  const auto give_up = [&] {
    if (kCtas == 2 && lane < 2) store_at(smem_of_rank(&sm.gave_up, lane), 1);
  };
  // Step kb of a tile to stage st, by one thread.
  const auto load_stage = [&](const Tile& tl, int kb, int st) {
    const int bn = work.bn(p, tl), bn_own = bn / kCtas;  // columns of B, and this CTA's
    const int m0 = tl.m * kRows + rank * kBM, n0 = tl.n * bn + rank * bn_own;
    const uint32_t stage_bytes = kCtas * ((kMode == kStats && kCtas == 1 ? p.a_rows * 128 : kABytes) + bn_own * 128);
    uint64_t* bar = &sm.full[st];
    const uint32_t pair_bar = kCtas == 2 ? smem_of_rank(bar, 0) : 0;  // the leader's
    const auto load = [&](void* dst, const CUtensorMap* map, int c0, int c1) {
      if (kCtas == 2)
        tma_load_2d_pair(dst, map, pair_bar, c0, c1);
      else
        tma_load_2d(dst, map, bar, c0, c1);
    };
    if (rank == 0) mbar_arrive_expect_tx(bar, stage_bytes);
    if (kMode == kStats || kMode == kGrad) {
      load(sm.a[st], &ma, kb * kBK, m0);
      load(sm.b[st], &mb, kb * kBK, p.v0 + n0);
    } else if (tl.dw) {
      for (int i = 0; i < 2; ++i) load(sm.a[st] + i * kBoxBytes, &mda, 0, (m0 / 64 + i) * p.n_pad + kb * kBK);
      if (kCtas == 2)
        load(sm.b[st], &mdb, kb * kBK, n0);
      else
        for (int i = 0; i < bn_own / 64; ++i) load(sm.b[st] + i * kBoxBytes, &mdb, n0 + 64 * i, kb * kBK);
    } else if (kCtas == 2) {
      for (int i = 0; i < 2; ++i) load(sm.a[st] + i * kBoxBytes, &ma, m0 + 64 * i, p.v0 + kb * kBK);
      load(sm.b[st], &mb, 0, kb * p.n_pad + n0);
    } else {
      load(sm.a[st], &ma, 0, kb * p.n_pad + m0);
      for (int i = 0; i < bn_own / 64; ++i) load(sm.b[st] + i * kBoxBytes, &mb, n0 + 64 * i, p.v0 + kb * kBK);
    }
  };
  if (warp == 0) {
    // ================================================================ TMA producer
    int fill = 0;
    bool ok = true;
    for (int j = 0, item; ok && (item = work.item(worker, workers, j)) >= 0; ++j) {
      const int t1 = work.last(p, item);
      for (int t = work.first(p, item); ok && t < t1; ++t) {
        const Tile tl = work.tile(p, item, t);
        for (int kb = tl.k0; kb < tl.k1; ++kb, ++fill) {
          const int st = fill % kStages;
          if (fill >= kStages && !warp_wait(&sm.empty[st], ((fill / kStages) - 1) & 1, abort, p.err, p.wait_ns)) {
            ok = false;
            break;
          }
          if (lane == 0) load_stage(tl, kb, st);
        }
      }
    }
    launch_dependents();
    // Teardown: every copy issued lands before the block exits. A single CTA waits for its
    // barriers; of a pair, whose copies complete on the leader's, each waits for the MMAs
    // that read its stages, and where something has given up both settle their accounts
    // behind the roles.
    if (kCtas == 2) {
      bool landed = ok;
      for (int s = 0; s < kStages; ++s) {
        const int n_s = fill > s ? (fill - s + kStages - 1) / kStages : 0;
        if (n_s && landed) landed = warp_wait(&sm.empty[s], (n_s - 1) & 1, abort, p.err, p.wait_ns);
      }
      if (lane < 2) store_at(smem_of_rank(&sm.loads[rank], lane), fill);  // here and in the other CTA
      if (!landed) give_up();
    } else if (lane == 0) {
      for (int s = 0; s < kStages; ++s) {
        const int n_s = fill > s ? (fill - s + kStages - 1) / kStages : 0;
        if (n_s) mbar_drain(&sm.full[s], (n_s - 1) & 1);
      }
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ================================================================ MMA issuer
    const auto commit = [](uint64_t* bar) {
      if (kCtas == 2)
        mma_commit_pair_elect(bar);
      else
        mma_commit_elect(bar);
    };
    // A step of 16 in K: 32 bytes of each row (K-major), or 16 rows of 128 bytes (MN-major:
    // single CTAs' B in back, g in dw, and a pair's weight in dh).
    constexpr bool b_mn = kMode == kBack && kCtas == 1;
    constexpr uint32_t b_step = b_mn ? 128 : 2;
    const uint64_t b_desc0 = sdesc_sw128(smem_u32(sm.b[0]), b_mn ? kBoxBytes : 16, 1024);
    int fill = 0, tile = 0;
    bool ok = true;
    for (int j = 0, item; ok && (item = work.item(worker, workers, j)) >= 0; ++j) {
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
        const bool a_mn = kMode == kBack && (kCtas == 2 || tl.dw);
        const uint32_t a_step = a_mn ? 128 : 2;
        const uint32_t idesc = idesc_bf16_f32(kRows, work.bn(p, tl), a_mn, b_mn);
        const uint64_t a_desc0 = sdesc_sw128(smem_u32(sm.a[0]), a_mn ? kBoxBytes : 16, 1024);
        for (int kb = tl.k0; kb < tl.k1; ++kb, ++fill) {
          const int st = fill % kStages;
          if (!warp_wait(&sm.full[st], (fill / kStages) & 1, abort, p.err, p.wait_ns)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t a_desc = a_desc0 + static_cast<uint32_t>(st) * (kABytes >> 4);
          const uint64_t b_desc = b_desc0 + static_cast<uint32_t>(st) * (kBBytes >> 4);
          // Of dw's last step only the scored rows' 16s: past those g is 0, the hidden states are
          // not.
          const int kks = kMode == kBack && tl.dw && kb == tl.k1 - 1 ? work.k_tail : kBK / 16;
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk) {
            if (kMode == kBack && kk >= kks) break;
            if (kCtas == 2)
              mma_ss_pair_elect(d_tmem, a_desc + kk * a_step, b_desc + kk * b_step, idesc, (kb > tl.k0 || kk > 0) ? 1u : 0u);
            else
              mma_ss_elect(d_tmem, a_desc + kk * a_step, b_desc + kk * b_step, idesc, (kb > tl.k0 || kk > 0) ? 1u : 0u);
          }
          commit(&sm.empty[st]);
        }
        if (!ok) break;
        commit(&sm.acc_full[acc]);
      }
    }
    // In this CTA alone: the other one does not wait for it, and may be gone when it arrives.
    if (kCtas == 2)
      mma_commit_leader_elect(&sm.done);
    else
      mma_commit_elect(&sm.done);
    mbar_drain(&sm.done, 0);
    if (!ok) give_up();
    if (kCtas == 2 && lane < 2) {
      store_at(smem_of_rank(&sm.mma_steps, lane), fill);
      store_at(smem_of_rank(&sm.mma_tiles, lane), tile);
    }
    __syncwarp();
  } else if (warp >= kEpiWarp0) {
    // ================================================================ epilogue
    // Two warps for each 32 rows, which take the tile's groups of 64 columns in turn. (One
    // warp: with d = 200 or 512 the epilogue is what a tile waits for.)
    const int qw = warp & 3;                         // TMEM lanes 32 qw .. 32 qw + 31
    const int half = (warp - kEpiWarp0) >> 2;
    const int t_row = qw * 32 + lane;                // row within the tile
    const uint32_t lane_base = static_cast<uint32_t>(qw * 32) << 16;
    uint8_t* buf = sm.out[warp - kEpiWarp0];
    const auto release = [&](int acc) {  // every column of the accumulator has been read
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (kCtas == 2)
          mbar_arrive_at(smem_of_rank(&sm.acc_empty[acc], 0));
        else
          mbar_arrive(&sm.acc_empty[acc]);
      }
    };
    const float scale = kMode == kStats ? 1.f : p.plan->scale;
    int tile = 0;
    bool ok = true;
    for (int j = 0, item; ok && (item = work.item(worker, workers, j)) >= 0; ++j) {
      const int t1 = work.last(p, item);
      float m = -INFINITY, s = 0.f;  // stats: over the item's tiles
      int target = -1;
      float lse2 = 0.f, dloss = 0.f;
      if (kMode == kStats || kMode == kGrad) {
        const int row = (item % work.row_blocks) * kRows + rank * kBM + t_row;
        target = p.target[row];
        if (kMode == kGrad) {
          lse2 = p.lse2[row];
          dloss = p.dloss[row] / scale;
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
        const int row = tl.m * kRows + rank * kBM + t_row;
        float ts = 0.f;  // stats: this tile's terms, relative to m
        const int groups = work.bn(p, tl) / 64;
        if (half >= groups) release(acc);
        // 64 columns at a time: two loads and one wait, and arithmetic enough without a
        // dependence that two warps a scheduler keep it busy.
#pragma unroll 1
        for (int g = half; g < groups; g += 2) {
          float x[64];
          {
            uint32_t v0[32], v1[32];
            tmem_ld32(base + 64 * g, v0);
            tmem_ld32(base + 64 * g + 32, v1);
            tmem_wait_ld(v0);
            tmem_wait_ld(v1);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              x[e] = __uint_as_float(v0[e]);
              x[32 + e] = __uint_as_float(v1[e]);
            }
          }
          if (g + 2 >= groups) release(acc);
          const int col0 = (kMode == kGrad ? p.v0 : 0) + tl.n * work.bn(p, tl) + 64 * g;
          if (kMode == kStats) {
            if (static_cast<unsigned>(target - col0) < 64u) {
              float xt = x[0];
#pragma unroll
              for (int e = 1; e < 64; ++e)
                if (target - col0 == e) xt = x[e];
              p.x_target[row] = xt;
            }
            if (col0 + 64 > p.V) {
#pragma unroll
              for (int e = 0; e < 64; ++e)
                if (col0 + e >= p.V) x[e] = -INFINITY;
            }
            float cm[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              cm[k] = fmax3(x[16 * k], x[16 * k + 1], x[16 * k + 2]);
#pragma unroll
              for (int e = 3; e < 15; e += 2) cm[k] = fmax3(cm[k], x[16 * k + e], x[16 * k + e + 1]);
              cm[k] = fmaxf(cm[k], x[16 * k + 15]);
            }
            const float top = fmaxf(fmax3(cm[0], cm[1], cm[2]), cm[3]);
            if (top > m) {
              const float a = m == -INFINITY ? 1.f : ex2_approx((m - top) * kLog2e);  // nothing, or a NaN, yet
              s *= a;
              ts *= a;
              m = top;
            }
            const float ml = m == -INFINITY ? 0.f : m * kLog2e;
            const float2 k2 = make_float2(kLog2e, kLog2e), n2 = make_float2(-ml, -ml);
            float2 sum[4] = {};
#pragma unroll
            for (int e = 0; e < 64; e += 2) {
              const float2 y = ffma2(make_float2(x[e], x[e + 1]), k2, n2);
              sum[e / 2 % 4] = fadd2(sum[e / 2 % 4], make_float2(ex2_approx(y.x), ex2_approx(y.y)));
            }
            const float2 both = fadd2(fadd2(sum[0], sum[1]), fadd2(sum[2], sum[3]));
            ts += both.x + both.y;
          } else {
            if (kMode == kGrad) {
              const float2 k2 = make_float2(kLog2e, kLog2e), n2 = make_float2(-lse2, -lse2);
#pragma unroll
              for (int e = 0; e < 64; e += 2) {
                const float2 y = ffma2(make_float2(x[e], x[e + 1]), k2, n2);
                x[e] = ex2_approx(y.x);
                x[e + 1] = ex2_approx(y.y);
              }
              if (static_cast<unsigned>(target - col0) < 64u) {
#pragma unroll
                for (int e = 0; e < 64; ++e) x[e] -= target - col0 == e ? 1.f : 0.f;
                float gt = 0.f;
#pragma unroll
                for (int e = 0; e < 64; ++e) take_if(target - col0, e, x[e], &gt);
                gt *= dloss;
                const float rest = gt - __bfloat162float(__float2bfloat16_rn(gt));
                p.rest[row] = fabsf(rest) < INFINITY ? rest : 0.f;
              }
              const float2 d2 = make_float2(dloss, dloss);
#pragma unroll
              for (int e = 0; e < 64; e += 2) {
                const float2 y = fmul2(make_float2(x[e], x[e + 1]), d2);
                x[e] = y.x;
                x[e + 1] = y.y;
              }
              if (col0 + 64 > p.V) {
#pragma unroll
                for (int e = 0; e < 64; ++e)
                  if (col0 + e >= p.V) x[e] = 0.f;
              }
              if (target < 0) {  // rows behind the scored ones hold anything: their g is 0
#pragma unroll
                for (int e = 0; e < 64; ++e) x[e] = 0.f;
              }
            }
            if (kMode == kBack && tl.dw) {
              const float2 s2 = make_float2(scale, scale);
#pragma unroll
              for (int e = 0; e < 64; e += 2) {
                const float2 y = fmul2(make_float2(x[e], x[e + 1]), s2);
                x[e] = y.x;
                x[e + 1] = y.y;
              }
            }
            if (kMode == kBack && tl.k1 == tl.k0) {  // no scored row: nothing was multiplied
#pragma unroll
              for (int e = 0; e < 64; ++e) x[e] = 0.f;
            }
            const int r0 = tl.m * kRows + rank * kBM + qw * 32;
            uint8_t* dst = buf + lane * 128;
            const auto filled = [&](auto store) {
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) {
                store();
                bulk_commit();
              }
            };
            const auto free_again = [&] {  // the store before has left the buffer
              if (lane == 0) bulk_wait_read<0>();
              __syncwarp();
            };
            if (kMode == kBack && !tl.dw) {
              // 32 columns of fp32 a buffer. The splits' sums lie behind each other: a pair's, whose
              // tile is transposed, along the columns.
              const int behind = tl.split * work.row_blocks * kRows;
              const int x0 = col0 + (kCtas == 2 ? behind : 0), y = r0 + (kCtas == 2 ? 0 : behind);
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                free_again();
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  *reinterpret_cast<float4*>(dst + ((e ^ (lane & 7)) << 4)) =
                      make_float4(x[32 * c + 4 * e], x[32 * c + 4 * e + 1], x[32 * c + 4 * e + 2], x[32 * c + 4 * e + 3]);
                filled([&] {
                  if (kCtas == 1 && x0 + 32 * c >= p.dh_cols) return;
                  if (!p.add)
                    tma_store_2d(&mo, buf, x0 + 32 * c, y);
                  else if (tl.k1 > tl.k0)
                    tma_add_2d(&mo, buf, x0 + 32 * c, y);
                });
              }
            } else {
              free_again();
#pragma unroll
              for (int e = 0; e < 8; ++e)
                *reinterpret_cast<uint4*>(dst + ((e ^ (lane & 7)) << 4)) =
                    make_uint4(pack_bf16x2(x[8 * e], x[8 * e + 1]), pack_bf16x2(x[8 * e + 2], x[8 * e + 3]),
                               pack_bf16x2(x[8 * e + 4], x[8 * e + 5]), pack_bf16x2(x[8 * e + 6], x[8 * e + 7]));
              filled([&] {
                if (kMode == kGrad)
                  tma_store_2d(&mo, buf, 0, (col0 - p.v0) / 64 * p.n_pad + r0);
                else if (p.v0 + r0 < p.dw_rows && col0 < p.dw_cols)
                  tma_store_2d(&mdo, buf, col0, p.v0 + r0);
              });
            }
          }
        }
        s += ts;
      }
      if (!ok) {
        give_up();
        break;
      }
      if (kMode == kStats)
        p.part[(static_cast<int64_t>(item) + static_cast<int64_t>(half) * work.items) * kRows + rank * kBM + t_row] = make_float2(m, s);
    }
    if (kMode != kStats && lane == 0) bulk_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  if (kCtas == 2)
    cg::this_cluster().sync();  // neither CTA's memory goes while the pair's copies and MMAs may use it
  else
    __syncthreads();
  if (kCtas == 2 && sm.gave_up) {  // (the same in both)
    if (threadIdx.x == 0) {
      // The commits that arrive here, one of a barrier on its way at most: the next one needs
      // what has waited for it.
      const int steps = sm.mma_steps, tiles = sm.mma_tiles;
      bool came = true;
      for (int s = 0; s < kStages; ++s) {
        const int n_s = steps > s ? (steps - s + kStages - 1) / kStages : 0;
        if (n_s && came) came = mbar_drain(&sm.empty[s], (n_s - 1) & 1);
      }
      for (int i = 0; i < 2; ++i) {
        const int n_i = tiles > i ? (tiles - i + 1) / 2 : 0;
        if (n_i && came) came = mbar_drain(&sm.acc_full[i], (n_i - 1) & 1);
      }
      // The CTA behind loads what the other one has loaded (into stages that are free, or the
      // other one's would not have been), so that every step's barrier in the leader gets
      // all its bytes; there their number is waited for.
      const int mine = sm.loads[rank], both = max(sm.loads[0], sm.loads[1]);
      int at = 0;
      for (int j = 0, item; at < both && (item = work.item(worker, workers, j)) >= 0; ++j) {
        const int t1 = work.last(p, item);
        for (int t = work.first(p, item); at < both && t < t1; ++t) {
          const Tile tl = work.tile(p, item, t);
          for (int kb = tl.k0; at < both && kb < tl.k1; ++kb, ++at)
            if (at >= mine) load_stage(tl, kb, at % kStages);
        }
      }
      if (rank == 0)
        for (int s = 0; s < kStages; ++s) {
          const int n_s = both > s ? (both - s + kStages - 1) / kStages : 0;
          if (n_s && came) came = mbar_drain(&sm.full[s], (n_s - 1) & 1);
        }
    }
    __syncwarp();
    cg::this_cluster().sync();
  }
  if (warp == 1) {
    tc_fence_after();
    if (kCtas == 2)
      tmem_dealloc_pair(tmem, kTmemCols);
    else
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
  int* origin;          // pairs' gradients: the row of each scored one
  __nv_bfloat16* d_hidden;  // pairs' gradients: 0 for rows that are not scored (may be null)
  int64_t s_dhidden;
  float* loss;          // loss only: 0 for rows that are not scored
  float* lse_out;
  bool gradients;
  int pair_rows;        // the scored rows from which CTAs work in pairs, 0: never
  struct Form {
    int block_rows;     // rows of a tile
    int tiles, workers, dw_tiles;  // gradients: what the K splits of dh depend on, with kblocks and max_rows
  } form[2];            // single CTAs, pairs
  int kblocks, max_rows;
};

constexpr int kGatherThreads = 256;

// The K splits of dh that end the launch first: no worker is done before its rounds of dh,
// nor before its share of dh and dw. A lane of a warp looks at two numbers of splits (one
// thread at all of them: 8 us).
__device__ int choose_splits(const GatherParams& p, const GatherParams::Form& f, int n) {
  const int lane = threadIdx.x & 31, blocks = (n + f.block_rows - 1) / f.block_rows;
  const float c_dw = dw_cost((n + kBK - 1) / kBK);
  float best = INFINITY;
  int splits = 1;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = lane + 32 * k + 1;
    const bool fits = s == 1 || (s <= p.kblocks && blocks <= p.max_rows / f.block_rows / s);
    const int dh = blocks * f.tiles * s, rounds = (dh + f.workers - 1) / f.workers;
    const float c_dh = dh_cost((p.kblocks + s - 1) / s, max(blocks, 1));
    const float share = (static_cast<float>(dh) * c_dh + static_cast<float>(f.dw_tiles) * c_dw) / static_cast<float>(f.workers);
    const float cost = fits ? fmaxf(static_cast<float>(rounds) * c_dh, share) : INFINITY;
    if (cost < best) {
      best = cost;
      splits = s;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float c = __shfl_xor_sync(0xffffffffu, best, o);
    const int s = __shfl_xor_sync(0xffffffffu, splits, o);
    if (c < best || (c == best && s < splits)) {
      best = c;
      splits = s;
    }
  }
  return splits;
}

__device__ __forceinline__ void store_bf16x8(__nv_bfloat16* dst, uint4 v, bool aligned) {
  if (aligned) {
    *reinterpret_cast<uint4*>(dst) = v;
    return;
  }
  unsigned short* e = reinterpret_cast<unsigned short*>(dst);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    e[2 * k] = static_cast<unsigned short>(w[k] & 0xFFFFu);
    e[2 * k + 1] = static_cast<unsigned short>(w[k] >> 16);
  }
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
// last one knows their number and what has to be behind them.
__global__ void __launch_bounds__(kGatherThreads) loss_gather_kernel(const GatherParams p) {
  __shared__ int sums[kGatherThreads / 32];
  __shared__ int source[kGatherThreads], others[kGatherThreads];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  wait_for_previous();
  launch_dependents();
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
      if (p.origin) p.origin[before + at] = static_cast<int>(r);
      if (p.to_lse2) {
        const float dl = p.dloss[r];
        p.to_lse2[before + at] = p.lse[r] * kLog2e;
        p.to_dloss[before + at] = dl;
        if (before + at == 0) {  // 1 where there is no such number
          const uint32_t bits = __float_as_uint(dl), exponent = bits >> 23 & 0xFFu;
          p.plan->scale = exponent == 0 || exponent == 255 ? 1.f : __uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u);
        }
      }
    }
    if (r < r1) {
      if (!on) others[threadIdx.x - at] = static_cast<int>(threadIdx.x);
      p.place[r] = on ? before + at : -1;
      if (!on && p.loss) {
        p.loss[r] = 0.f;
        p.lse_out[r] = 0.f;
      }
    }
    __syncthreads();
    constexpr int kLoads = 4;  // of 16 bytes, in flight
    const int64_t words = static_cast<int64_t>(total) * vecs;
    for (int64_t i0 = threadIdx.x; i0 < words; i0 += kGatherThreads * kLoads) {
      uint4 v[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        const int64_t i = i0 + k * kGatherThreads;
        v[k] = make_uint4(0, 0, 0, 0);
        if (i >= words) continue;
        const int row = static_cast<int>(i / vecs), col = static_cast<int>(i - static_cast<int64_t>(row) * vecs);
        if (col >= full) continue;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.hidden) + (base + source[row]) * p.s_hidden + 8 * col;
        if (aligned) {
          v[k] = *reinterpret_cast<const uint4*>(src);
        } else {
          const unsigned short* e = reinterpret_cast<const unsigned short*>(src);
          v[k] = make_uint4(e[0] | static_cast<uint32_t>(e[1]) << 16, e[2] | static_cast<uint32_t>(e[3]) << 16,
                            e[4] | static_cast<uint32_t>(e[5]) << 16, e[6] | static_cast<uint32_t>(e[7]) << 16);
        }
      }
#pragma unroll
      for (int k = 0; k < kLoads; ++k)
        if (i0 + k * kGatherThreads < words) p.to_hidden[static_cast<int64_t>(before) * vecs + i0 + k * kGatherThreads] = v[k];
    }
    if (p.d_hidden) {
      const int rows = static_cast<int>(r1 - base < kGatherThreads ? r1 - base : kGatherThreads) - total;
      const bool whole = ((reinterpret_cast<uintptr_t>(p.d_hidden) | static_cast<uintptr_t>(p.s_dhidden * 2)) & 15) == 0;
      for (int64_t i = threadIdx.x; i < static_cast<int64_t>(rows) * full; i += kGatherThreads) {
        const int row = static_cast<int>(i / full), col = static_cast<int>(i - static_cast<int64_t>(row) * full);
        store_bf16x8(p.d_hidden + (base + others[row]) * p.s_dhidden + 8 * col, make_uint4(0, 0, 0, 0), whole);
      }
    }
    before += total;
  }
  if (blockIdx.x != gridDim.x - 1) return;
  const int n = before, end = (n + 2 * kBM - 1) / (2 * kBM) * (2 * kBM);
  if (warp == 0) {
    const int pairs = p.pair_rows && pairs_pay(n, p.pair_rows, p.gradients);
    const int splits = p.gradients ? choose_splits(p, p.form[pairs], n) : 1;
    if (lane == 0) {
      p.plan->n = n;
      p.plan->pairs = pairs;
      p.plan->splits = splits;
    }
  }
  for (int r = n + threadIdx.x; r < end; r += kGatherThreads) {
    p.to_target[r] = -1;
    if (p.to_lse2) p.to_lse2[r] = p.to_dloss[r] = 0.f;
  }
  if (!p.to_lse2) return;
  // dw's last 16 rows multiply the hidden states behind the scored ones by 0.
  const int64_t rows_end = (n + 15) / 16 * 16;
#pragma unroll 4
  for (int64_t i = static_cast<int64_t>(n) * vecs + threadIdx.x; i < rows_end * vecs; i += kGatherThreads)
    p.to_hidden[i] = make_uint4(0, 0, 0, 0);
}

// The hidden states of the scored rows transposed, [d_pad, n_pad], for a pair's dw: 64 x 64
// a CTA (what lies behind the last 64 rows is left as it is).
constexpr int kTransposeThreads = 256;
__global__ void __launch_bounds__(kTransposeThreads)
    loss_transpose_kernel(const Plan* plan, const uint4* hidden, int d_pad, int n_pad, uint4* out) {
  __shared__ uint32_t tile[64][33];  // rows of 32 pairs of columns
  wait_for_previous();
  launch_dependents();
  const int r0 = blockIdx.x * 64, d0 = blockIdx.y * 64, r = threadIdx.x >> 3, v = threadIdx.x & 7;
  if (!plan->pairs || r0 >= plan->n) return;
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const uint4 u = hidden[(static_cast<int64_t>(r0 + r + i) * d_pad + d0) / 8 + v];
    tile[r + i][4 * v] = u.x;
    tile[r + i][4 * v + 1] = u.y;
    tile[r + i][4 * v + 2] = u.z;
    tile[r + i][4 * v + 3] = u.w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int c = r + i, shift = (c & 1) * 16;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k] = (tile[8 * v + 2 * k][c >> 1] >> shift & 0xFFFFu) | (tile[8 * v + 2 * k + 1][c >> 1] >> shift) << 16;
    out[(static_cast<int64_t>(d0 + c) * n_pad + r0) / 8 + v] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---------------------------------------------------------------- results

// Joins the parts of each scored row, a warp a row.
constexpr int kCombineThreads = 256;
__global__ void __launch_bounds__(kCombineThreads)
    loss_combine_kernel(const Plan* plan, const int* place, const float2* part, const float* x_target, int N, int parts_single,
                        int parts_pairs, float* loss, float* lse) {
  wait_for_previous();
  const int64_t r = (static_cast<int64_t>(blockIdx.x) * kCombineThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (r >= N) return;
  const int c = place[r];
  if (c < 0) return;  // written by the first launch
  const int block_rows = plan->pairs ? 2 * kBM : kBM, parts = plan->pairs ? parts_pairs : parts_single;
  const int64_t step = static_cast<int64_t>((plan->n + block_rows - 1) / block_rows) * block_rows;
  constexpr int kPer = (2 * kLossMaxParts + 31) / 32;
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

// What turns the sums of g weight into d_hidden: the rest of the target's g, and the scale.
struct Finish {
  const int* target;  // of each row (pairs: of each scored one)
  const float* rest;  // of each scored row
  const __nv_bfloat16* weight;
  int64_t s_weight;
};

// d_hidden: the splits' sums of each scored row, zeros for the others; four columns a
// thread, eight splits' loads in flight.
constexpr int kFinishThreads = 128;
__global__ void __launch_bounds__(kFinishThreads)
    loss_dhidden_kernel(const Plan* plan, const Finish f, const int* place, const float* part, int N, int d, int d_pad,
                        __nv_bfloat16* out, int64_t s_out, int aligned) {
  wait_for_previous();
  if (plan->pairs) return;
  const int vecs = d / 4, splits = plan->splits;
  const float scale = plan->scale;
  const int64_t step = static_cast<int64_t>((plan->n + kBM - 1) / kBM) * kBM * d_pad;
  const int64_t total = static_cast<int64_t>(N) * vecs;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kFinishThreads + threadIdx.x; i < total;
       i += static_cast<int64_t>(gridDim.x) * kFinishThreads) {
    const int64_t r = i / vecs;
    const int col = static_cast<int>(i - r * vecs) * 4, c = place[r], t = f.target[r];
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c >= 0) {
      const float* src = part + static_cast<int64_t>(c) * d_pad + col;
      const uint2 w = *reinterpret_cast<const uint2*>(f.weight + t * f.s_weight + col);
      const float rest = f.rest[c];
      for (int s = 0; s < splits; s += 8) {
        float4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          v[k] = s + k < splits ? *reinterpret_cast<const float4*>(src + (s + k) * step) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) a = make_float4(a.x + v[k].x, a.y + v[k].y, a.z + v[k].z, a.w + v[k].w);
      }
      a = make_float4(fmaf(rest, __uint_as_float(w.x << 16), a.x) * scale, fmaf(rest, __uint_as_float(w.x & 0xFFFF0000u), a.y) * scale,
                      fmaf(rest, __uint_as_float(w.y << 16), a.z) * scale, fmaf(rest, __uint_as_float(w.y & 0xFFFF0000u), a.w) * scale);
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

// The same from a pair's sums, [., columns] with a row for each column of d_hidden and the
// splits behind each other, whole blocks of rows apart: 32 rows x 64 columns a CTA.
constexpr int kTurnThreads = 256;
__global__ void __launch_bounds__(kTurnThreads)
    loss_dhidden_turn_kernel(const Plan* plan, const Finish f, const int* origin, const float* part, int d, int64_t columns,
                             __nv_bfloat16* out, int64_t s_out, int aligned) {
  __shared__ float tile[64][33];
  wait_for_previous();
  if (!plan->pairs) return;
  const int n = plan->n, splits = plan->splits, r0 = blockIdx.x * 32, d0 = blockIdx.y * 64;
  if (r0 >= n) return;
  const int64_t step = static_cast<int64_t>((n + 2 * kBM - 1) / (2 * kBM)) * (2 * kBM);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
  const bool on = r0 + r < n && d0 + c < d;
  uint4 u = make_uint4(0, 0, 0, 0);
  float rest = 0.f;
  if (on) {
    u = *reinterpret_cast<const uint4*>(f.weight + f.target[r0 + r] * f.s_weight + d0 + c);
    rest = f.rest[r0 + r];
  }
  float a[8] = {};
  for (int s = 0; s < splits; ++s) {
    const float* src = part + (d0 + warp) * columns + s * step + r0 + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] += src[8 * i * columns];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) tile[warp + 8 * i][lane] = a[i];
  __syncthreads();
  if (!on) return;
  const float scale = plan->scale;
  uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    w[k] = pack_bf16x2(fmaf(rest, __uint_as_float(w[k] << 16), tile[c + 2 * k][r]) * scale,
                       fmaf(rest, __uint_as_float(w[k] & 0xFFFF0000u), tile[c + 2 * k + 1][r]) * scale);
  store_bf16x8(out + static_cast<int64_t>(origin[r0 + r]) * s_out + d0 + c, make_uint4(w[0], w[1], w[2], w[3]), aligned);
}

// ---------------------------------------------------------------- host side

int sm_count() {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

// Columns of a tile: 256, or 128 or 64 (single CTAs) where 256 leave SMs without a tile or
// much of the last tile empty (narrow tiles read their other operand more often: a column
// counts 1.12 and 1.36 times, as in the projection's own choice). With one worker: by the
// last tile alone (dw has tiles enough, dh is split).
int choose_bn(int64_t cols, int64_t row_tiles, int workers, int ctas) {
  int best = 256;
  double best_cost = 1e300;
  for (int bn = 256; bn >= 64 * ctas; bn /= 2) {
    const int64_t tiles = (cols + bn - 1) / bn * row_tiles, rounds = (tiles + workers - 1) / workers;
    const double cost = static_cast<double>(rounds) * (bn / 256.0 * 0.88 + 0.12);
    if (cost < best_cost - 1e-9) {
      best_cost = cost;
      best = bn;
    }
  }
  return best;
}

// The maps of a launch: operands and result, and back's of dw.
struct Maps {
  CUtensorMap a, b, out, dw_a, dw_b, dw_out;
};

template <int kMode, int kCtas>
int launch_product(const Maps& m, const Params& p, int64_t items, int workers, cudaStream_t stream) {
  const auto kernel = loss_product_kernel<kMode, kCtas>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<kCtas>()));
  const int64_t run = items < workers ? items : workers;
  if (e == cudaSuccess)
    e = launch_overlapped(kernel, dim3(static_cast<unsigned>(run * kCtas)), kThreads, smem_bytes<kCtas>(), stream, kCtas, true, m.a,
                          m.b, m.out, m.dw_a, m.dw_b, m.dw_out, p);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "projection loss launch: %s", cudaGetErrorString(e));
}

template <int kMode>
int launch_product(int ctas, const Maps& m, const Params& p, int64_t items, int workers, cudaStream_t stream) {
  return ctas == 2 ? launch_product<kMode, 2>(m, p, items, workers, stream) : launch_product<kMode, 1>(m, p, items, workers, stream);
}

// CTAs that share a tile, and how many such groups run at once. Pairs: none where the device
// has no place for them.
struct Team {
  int ctas, workers;
};

Team team_of(int ctas) {
  const int sms = sm_count();
  if (ctas == 1) return {1, sms};
  const auto kernel = loss_product_kernel<kBack, 2>;  // the same shared memory in every mode
  int pairs = 0;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<2>())) == cudaSuccess)
    pairs = active_clusters(reinterpret_cast<const void*>(kernel), 2, kThreads, smem_bytes<2>());
  if (pairs <= 0) cudaGetLastError();
  return {2, pairs < sms / 2 ? pairs : sms / 2};
}

// Places of the workspace, from its start.
struct Layout {
  int64_t n_pad, d_pad;
  size_t plan, place, target, lse2, dloss, rest, hidden, x_target, part, origin, turned, sums, g;  // byte offsets
  int64_t sums_rows;  // gradients: rows of fp32 sums (pairs: columns, of d_rows rows)
  int64_t d_rows;
};

size_t take(size_t* at, size_t bytes) {
  const size_t here = *at;
  *at += (bytes + 255) / 256 * 256;
  return here;
}

Layout layout_of(int64_t N, int64_t d, bool grad) {
  Layout l = {};
  l.n_pad = (N + 2 * kBM - 1) / (2 * kBM) * (2 * kBM);
  l.d_pad = (d + kBK - 1) / kBK * kBK;
  size_t at = 0;
  l.plan = take(&at, sizeof(Plan));
  l.place = take(&at, N * 4);
  l.target = take(&at, l.n_pad * 4);
  l.hidden = take(&at, l.n_pad * l.d_pad * 2);
  if (!grad) {
    l.x_target = take(&at, l.n_pad * 4);
    l.part = take(&at, static_cast<size_t>(2 * kLossMaxParts) * l.n_pad * 8);
  } else {
    l.lse2 = take(&at, l.n_pad * 4);
    l.dloss = take(&at, l.n_pad * 4);
    l.rest = take(&at, l.n_pad * 4);
    if (pairs_have_room(N, d)) {
      l.origin = take(&at, l.n_pad * 4);
      l.turned = take(&at, l.n_pad * l.d_pad * 2);
    }
    // Room for splits of dh: up to 32 of them, 192 MB, and one in any case.
    l.d_rows = (d + 2 * kBM - 1) / (2 * kBM) * (2 * kBM);
    const int64_t most = (int64_t{192} << 20) / (l.d_rows * 4) / (2 * kBM) * (2 * kBM);
    l.sums_rows = 32 * l.n_pad < most ? 32 * l.n_pad : most;
    if (l.sums_rows < l.n_pad) l.sums_rows = l.n_pad;
    l.sums = take(&at, static_cast<size_t>(l.sums_rows) * l.d_rows * 4);
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
  // No more CTAs than run at once: every CTA counts the rows before its own.
  int64_t rows = 1;
  while (a.N > rows * 1024) rows *= 2;
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
  int64_t cols = piece > all ? all : piece > 0 ? (piece + 255) / 256 * 256 : (int64_t{1} << 31) / (l.n_pad * 2) / 256 * 256;
  if (piece <= 0 && cols < 1024) cols = 1024;
  if (cols > all) cols = all;
  return l.g + static_cast<size_t>(l.n_pad) * cols * 2;
}

int launch_loss(const LossArgs& a, cudaStream_t stream) {
  const Layout l = layout_of(a.N, a.d, false);
  const int from = pair_rows(a.N, a.V, a.d, false);
  const Team teams[2] = {team_of(1), from ? team_of(2) : Team{2, 0}};
  const bool either = teams[1].workers > 0;
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  Params p = common_params(a, l);
  p.either = either;
  p.kblocks = static_cast<int>(l.d_pad / kBK);
  p.part = reinterpret_cast<float2*>(ws + l.part);
  p.x_target = reinterpret_cast<float*>(ws + l.x_target);
  p.a_rows = a.N < kBM ? static_cast<int>((a.N + 7) / 8 * 8) : kBM;
  // Single CTAs, and pairs where they may work; what can be refused, before the first launch.
  struct Form {
    int64_t row_blocks;
    int bn, tiles, parts;
    Maps maps;
  } forms[2] = {};
  int st;
  for (int i = 0; i <= (either ? 1 : 0); ++i) {
    Form& f = forms[i];
    const int ctas = teams[i].ctas, block_rows = kBM * ctas;
    f.row_blocks = (a.N + block_rows - 1) / block_rows;
    f.bn = choose_bn(a.V, f.row_blocks, teams[i].workers, ctas);
    f.tiles = static_cast<int>((a.V + f.bn - 1) / f.bn);
    f.parts = f.tiles < kLossMaxParts ? f.tiles : kLossMaxParts;
    if ((st = make_matrix_map(&f.maps.a, ws + l.hidden, true, l.n_pad, l.d_pad, l.d_pad, p.a_rows)) != DLM_OK) return st;
    if ((st = make_matrix_map(&f.maps.b, a.weight, true, a.V, a.d, a.s_weight, f.bn / ctas)) != DLM_OK) return st;
  }
  GatherParams g = {};
  g.pair_rows = either ? from : 0;
  g.loss = a.loss;
  g.lse_out = a.lse_out;
  if ((st = launch_gather(a, l, g, stream)) != DLM_OK) return st;
  for (int i = 0; i <= (either ? 1 : 0); ++i) {
    const Form& f = forms[i];
    p.bn = f.bn;
    p.tiles = f.tiles;
    p.parts = f.parts;
    if ((st = launch_product<kStats>(teams[i].ctas, f.maps, p, f.parts * f.row_blocks, teams[i].workers, stream)) != DLM_OK) return st;
  }
  const cudaError_t e = launch_overlapped(
      loss_combine_kernel, dim3(static_cast<unsigned>((a.N * 32 + kCombineThreads - 1) / kCombineThreads)), kCombineThreads, 0, stream,
      1, true, p.plan, reinterpret_cast<const int*>(ws + l.place), static_cast<const float2*>(p.part),
      static_cast<const float*>(p.x_target), static_cast<int>(a.N), 2 * forms[0].parts, 2 * forms[1].parts, a.loss, a.lse_out);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "loss combine launch: %s", cudaGetErrorString(e));
}

int launch_loss_grad(const LossArgs& a, cudaStream_t stream) {
  const Layout l = layout_of(a.N, a.d, true);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  const int64_t all = (a.V + 255) / 256 * 256;
  int64_t cols = static_cast<int64_t>((a.workspace_bytes - l.g) / (static_cast<size_t>(l.n_pad) * 2)) / 256 * 256;
  // g lies in panels of 64 columns, whose rows follow each other: a box of any operand is
  // one run of memory. Their number times n_pad is a coordinate.
  const int64_t most_cols = int64_t{0x7FFFFF00} / l.n_pad * 64 / 256 * 256;
  if (cols > most_cols) cols = most_cols;
  if (cols > all) cols = all;
  const int64_t first = cols < a.V ? cols : a.V, panel_rows = l.n_pad * (cols / 64);

  // Single CTAs, and pairs where they may work.
  struct Form {
    Team team;
    int64_t row_blocks;
    int bn_d, bn_v, d_tiles, dh_tiles;
    Maps grad, back;
  } forms[2] = {};
  forms[0].team = team_of(1);
  const int from = pair_rows(a.N, a.V, a.d, true);
  forms[1].team = from ? team_of(2) : Team{2, 0};
  const bool either = forms[1].team.workers > 0;
  GatherParams g = {};
  int st;
  for (int i = 0; i <= (either ? 1 : 0); ++i) {
    Form& f = forms[i];
    const bool pairs = i == 1;
    const int ctas = f.team.ctas, block_rows = kBM * ctas;
    f.row_blocks = (a.N + block_rows - 1) / block_rows;
    f.bn_d = choose_bn(a.d, 1, 1, ctas);
    f.bn_v = choose_bn(first, f.row_blocks, f.team.workers, ctas);
    f.d_tiles = static_cast<int>((a.d + f.bn_d - 1) / f.bn_d);
    f.dh_tiles = pairs ? static_cast<int>(l.d_rows / (2 * kBM)) : f.d_tiles;
    g.form[i] = {block_rows, f.dh_tiles, f.team.workers,
                 a.d_weight ? static_cast<int>((first + block_rows - 1) / block_rows) * f.d_tiles : 0};
    Maps &grad = f.grad, &back = f.back;
    if ((st = make_matrix_map(&grad.a, ws + l.hidden, true, l.n_pad, l.d_pad, l.d_pad, kBM)) != DLM_OK) return st;
    if ((st = make_matrix_map(&grad.b, a.weight, true, a.V, a.d, a.s_weight, f.bn_v / ctas)) != DLM_OK) return st;
    if ((st = make_matrix_map(&grad.out, ws + l.g, true, panel_rows, 64, 64, 32)) != DLM_OK) return st;
    // dh: g times the weight, or, a pair's, the weight transposed times g transposed.
    if ((st = make_matrix_map(pairs ? &back.b : &back.a, ws + l.g, true, panel_rows, 64, 64, kBM)) != DLM_OK) return st;
    if ((st = make_matrix_map(pairs ? &back.a : &back.b, a.weight, true, a.V, a.d, a.s_weight, 64)) != DLM_OK) return st;
    st = pairs ? make_matrix_map(&back.out, ws + l.sums, false, l.d_rows, l.sums_rows, l.sums_rows, 32)
               : make_matrix_map(&back.out, ws + l.sums, false, l.sums_rows, l.d_pad, l.d_pad, 32);
    if (st != DLM_OK) return st;
    if ((st = make_matrix_map(&back.dw_a, ws + l.g, true, panel_rows, 64, 64, 64)) != DLM_OK) return st;
    st = pairs ? make_matrix_map(&back.dw_b, ws + l.turned, true, l.d_pad, l.n_pad, l.n_pad, f.bn_d / 2)
               : make_matrix_map(&back.dw_b, ws + l.hidden, true, l.n_pad, l.d_pad, l.d_pad, 64);
    if (st != DLM_OK) return st;
    if (a.d_weight && (st = make_matrix_map(&back.dw_out, a.d_weight, true, a.V, a.d, a.s_dweight, 32)) != DLM_OK) return st;
  }

  g.gradients = true;
  g.pair_rows = either ? from : 0;
  g.lse = a.lse;
  g.dloss = a.dloss;
  g.to_lse2 = reinterpret_cast<float*>(ws + l.lse2);
  g.to_dloss = reinterpret_cast<float*>(ws + l.dloss);
  g.kblocks = static_cast<int>((first + kBK - 1) / kBK);
  g.max_rows = l.sums_rows > 0x7FFFFFFF ? 0x7FFFFFFF : static_cast<int>(l.sums_rows);
  if (either) {
    g.origin = reinterpret_cast<int*>(ws + l.origin);
    g.d_hidden = static_cast<__nv_bfloat16*>(a.d_hidden);
    g.s_dhidden = a.s_dhidden;
  }
  if ((st = launch_gather(a, l, g, stream)) != DLM_OK) return st;

  Params p = common_params(a, l);
  p.either = either;
  p.n_pad = static_cast<int>(l.n_pad);
  p.lse2 = g.to_lse2;
  p.dloss = g.to_dloss;
  p.rest = reinterpret_cast<float*>(ws + l.rest);
  p.want_dw = a.d_weight != nullptr;
  p.want_dh = a.d_hidden != nullptr;
  p.dw_rows = p.V;
  p.dw_cols = static_cast<int>(a.d);
  p.dh_cols = static_cast<int>(l.d_pad);
  if (either && a.d_weight) {
    const cudaError_t e = launch_overlapped(
        loss_transpose_kernel, dim3(static_cast<unsigned>(l.n_pad / 64), static_cast<unsigned>(l.d_pad / 64)), kTransposeThreads, 0,
        stream, 1, true, p.plan, reinterpret_cast<const uint4*>(ws + l.hidden), static_cast<int>(l.d_pad), p.n_pad,
        reinterpret_cast<uint4*>(ws + l.turned));
    if (e != cudaSuccess) return fail(DLM_ERR_CUDA, "hidden states launch: %s", cudaGetErrorString(e));
  }
  for (int64_t v0 = 0; v0 < a.V; v0 += cols) {
    const int64_t vc = a.V - v0 < cols ? a.V - v0 : cols;
    p.v0 = static_cast<int>(v0);
    p.add = v0 > 0;
    for (int i = 0; i <= (either ? 1 : 0); ++i) {
      const Form& f = forms[i];
      p.kblocks = static_cast<int>(l.d_pad / kBK);
      p.bn = f.bn_v;
      p.tiles = static_cast<int>((vc + f.bn_v - 1) / f.bn_v);
      if ((st = launch_product<kGrad>(f.team.ctas, f.grad, p, p.tiles * f.row_blocks, f.team.workers, stream)) != DLM_OK) return st;
    }
    for (int i = 0; i <= (either ? 1 : 0); ++i) {
      const Form& f = forms[i];
      const int block_rows = kBM * f.team.ctas;
      p.bn = f.bn_d;
      p.tiles = f.d_tiles;
      p.dh_tiles = f.dh_tiles;
      p.parts = static_cast<int>((vc + block_rows - 1) / block_rows);
      p.kblocks = static_cast<int>((vc + kBK - 1) / kBK);
      if ((st = launch_product<kBack>(f.team.ctas, f.back, p, f.team.workers, f.team.workers, stream)) != DLM_OK) return st;
    }
  }
  if (!a.d_hidden) return DLM_OK;
  Finish f = {a.targets, p.rest, static_cast<const __nv_bfloat16*>(a.weight), a.s_weight};
  const int64_t vecs = a.N * (a.d / 4);
  const int64_t want = (vecs + kFinishThreads - 1) / kFinishThreads, most = static_cast<int64_t>(sm_count()) * 16;
  const uintptr_t place = reinterpret_cast<uintptr_t>(a.d_hidden) | static_cast<uintptr_t>(a.s_dhidden * 2);
  cudaError_t e = launch_overlapped(
      loss_dhidden_kernel, dim3(static_cast<unsigned>(want < most ? want : most)), kFinishThreads, 0, stream, 1, true, p.plan, f,
      reinterpret_cast<const int*>(ws + l.place), reinterpret_cast<const float*>(ws + l.sums), static_cast<int>(a.N),
      static_cast<int>(a.d), static_cast<int>(l.d_pad), static_cast<__nv_bfloat16*>(a.d_hidden), a.s_dhidden,
      (place & 7) == 0 ? 1 : 0);
  if (e == cudaSuccess && either) {
    f.target = p.target;
    e = launch_overlapped(
        loss_dhidden_turn_kernel, dim3(static_cast<unsigned>((a.N + 31) / 32), static_cast<unsigned>((a.d + 63) / 64)), kTurnThreads, 0,
        stream, 1, true, p.plan, f, g.origin, reinterpret_cast<const float*>(ws + l.sums), static_cast<int>(a.d), l.sums_rows,
        static_cast<__nv_bfloat16*>(a.d_hidden), a.s_dhidden, (place & 15) == 0 ? 1 : 0);
  }
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "hidden gradient launch: %s", cudaGetErrorString(e));
}

}  // namespace dlm
