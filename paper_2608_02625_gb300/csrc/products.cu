// Products of a feed-forward block on the tensor cores, their element-wise parts in the
// epilogue.
//
//   gated   out = act(x Wg^T) (x Wu^T)              a tile of rows of x against gate and up rows
//   cols    out = act(x W^T + bias) + residual      (also d x = dg Wg + du Wu + add, K in two runs)
//   rows    dW = dz^T x                             (also dWg and dWu: row tiles of one, then the other)
//
// One persistent kernel: two CTAs share a tile of 256 rows (cta_group::2), K steps of 64
// through a ring of 192 KB, two accumulators of up to 256 columns in tensor memory, so that a
// tile's epilogue runs under the next one's K loop. Warp 0 loads by TMA, warp 1 of the
// leader issues tcgen05.mma, warps 4-11 read the accumulators.
// Of what an MMA reads, B should be K-major (with an MN-major B the tensor pipe of pairs was
// busy 73 % of the cycles in the vocabulary projection's gradients, 90 % with a K-major one).
//   gated: A the rows of x; of B's 256 rows the leader loads 128 of the gate, the other CTA the
//          same 128 of up, so a thread of the epilogue has both of a feature in its lane
//   cols:  the result transposed: A the weight's rows (K-major as it lies), or, for d x, its
//          columns (MN-major), B the rows of x or dz. Lanes are output columns, so a warp's
//          stores, residuals and biases are 32 columns of a row side by side, and need no
//          alignment
//   rows:  A is dz's columns (MN-major), B x transposed once, before, to K-major
// The tensor pipe bounds it. 16384 rows, 2048 x 8192: gated (1.1 TFLOP) 631-645 us, cols 332-340, under
// the power cap (1.62-1.74 PFLOP/s); a gated block's d x and dW 590 each in single launches (1.86).
// Every wait is bounded; on expiry the kernel sets DLM_DEVERR_TIMEOUT, lets what it has on
// its way land (in both CTAs) and exits.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>

#include <cstdint>

#include "block_math.cuh"
#include "dlm_common.cuh"
#include "dlm_internal.h"
#include "dlm_tmap.h"
#include "products.h"

namespace cg = cooperative_groups;

namespace dlm {
namespace {

constexpr int kBM = 128;          // a CTA's rows of a tile = TMEM lanes
constexpr int kRows = 2 * kBM;    // a pair's
constexpr int kBK = 64;           // K of a stage: 128 bytes of bf16
constexpr int kMaxBN = 256;
constexpr int kThreads = 384;     // warp 0 TMA, warp 1 MMA, warps 4-11 epilogue
constexpr int kEpiWarp0 = 4, kEpiWarps = 8;
constexpr int kABytes = kBM * kBK * 2;
constexpr int kBoxBytes = 64 * 128;            // an MN-major box: 64 K rows of 64 columns
constexpr int kRing = 192 * 1024;              // 6 stages with B's half of 128 rows, 8 with one of 64
constexpr int kMaxStages = 8;
constexpr uint32_t kTmemCols = 2 * kMaxBN;     // two accumulators

enum Form { kGated, kCols, kColsTurned, kRowsForm };

struct Smem {
  alignas(1024) uint8_t ring[kRing];               // stages: this CTA's A and B
  alignas(1024) uint8_t out[kEpiWarps][32 * 128];  // per epilogue warp, 32 rows x 128 bytes
  uint64_t full[kMaxStages];   // stage loaded            (TMA -> MMA; in the leader)
  uint64_t empty[kMaxStages];  // stage read by its MMAs  (MMA -> TMA)
  uint64_t acc_full[2];     // accumulator complete    (MMA -> epilogue)
  uint64_t acc_empty[2];    // accumulator read out    (epilogue -> MMA; in the leader)
  uint64_t done;            // every MMA completed     (teardown; in the leader)
  uint32_t tmem_base;
  int abort;
  // In both CTAs: what each has loaded, what the leader's MMAs have committed, and whether a
  // role of either has given up.
  int loads[2], mma_steps, mma_tiles, gave_up;
};
constexpr size_t kSmemBytes = sizeof(Smem) + 1024;
static_assert(kSmemBytes <= 227 * 1024, "shared memory of a CTA");

struct Maps {
  CUtensorMap a[2], b[2];  // the operands; [1]: up (gated), the second run of K (cols), the second matrix (rows)
  CUtensorMap out[3];      // gated: out, gate, up;  rows: both results
};

struct Params {
  int row_tiles, col_tiles, first_tiles;  // first_tiles: rows: row tiles of the first matrix
  int kblocks, first_kblocks;             // K steps; those of the first run
  int bn;
  int act;
  int n, cols;          // extents of a result: rows and columns
  int keep;             // gated: gate and up too
  int wide;             // cols, from here on: rows of out, residual and pre are 16-byte aligned
  const void* bias;     // may be null
  int bias_bf16;
  const __nv_bfloat16* residual;  // may be null
  __nv_bfloat16* out;
  __nv_bfloat16* pre;   // may be null
  int64_t s_residual, s_out, s_pre;
  int* err;
  uint64_t wait_ns;
};

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* err, uint64_t budget_ns) {
  const bool ok = mbar_wait_for<true>(bar, parity, abort, err, budget_ns);
  return __all_sync(0xffffffffu, ok);
}

// A wait that asked before (`ready`, of the same phase): to look at a barrier takes some 170
// cycles, under which the step before is issued.
__device__ __forceinline__ bool warp_wait_if(bool ready, uint64_t* bar, uint32_t parity, volatile int* abort, int* err, uint64_t budget_ns) {
  if (!kCheckBounds && __all_sync(0xffffffffu, ready)) return true;
  return warp_wait(bar, parity, abort, err, budget_ns);
}

__device__ __forceinline__ void tma_store_2d(const void* tmap, const void* src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(smem_u32(src)), "r"(c0), "r"(c1)
               : "memory");
}

// The stages in turn (their number goes by the tile's columns: no divisions in the loops).
struct Ring {
  int stage = 0, round = 0;  // round: the parity of this pass over the stages
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) {
      stage = 0;
      round ^= 1;
    }
  }
};

// The t-th output tile. Tiles that run at the same time are about as many rows as columns, so
// that both operands are shared in L2: eight row tiles at a time, all column tiles of those.
struct Tile {
  int m, n;
};
constexpr int kGroup = 8;
__device__ __forceinline__ Tile tile_of(const Params& p, int t) {
  const int per = kGroup * p.col_tiles, g = t / per, rest = t - g * per;
  const int rows = min(kGroup, p.row_tiles - g * kGroup);
  return {g * kGroup + rest % rows, rest / rows};
}

template <int kForm>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ Maps maps, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int rank = static_cast<int>(blockIdx.x & 1);  // in the pair
  const int worker = static_cast<int>(blockIdx.x >> 1), workers = static_cast<int>(gridDim.x >> 1);
  const int tiles = p.row_tiles * p.col_tiles;
  constexpr bool a_mn = kForm == kColsTurned || kForm == kRowsForm;
  const int stage_bytes = kABytes + p.bn * 64, stages = kRing / stage_bytes;

  if (threadIdx.x == 32 * kEpiWarp0) {  // parameters, not memory that another kernel writes
    prefetch_tmap(&maps.a[0]);
    prefetch_tmap(&maps.b[0]);
    if (kForm == kGated || kForm == kRowsForm) prefetch_tmap(&maps.out[0]);
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.acc_full[i], 1);
      mbar_init(&sm.acc_empty[i], kEpiWarps * 2);
    }
    mbar_init(&sm.done, 1);
    sm.abort = 0;
    sm.gave_up = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    tmem_alloc_pair(&sm.tmem_base, kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cg::this_cluster().sync();  // the other CTA's barriers and tensor memory are there too
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  volatile int* abort = &sm.abort;
  wait_for_previous();
  // A role that ends early (a whole warp): see the end.
  const auto give_up = [&] {
    if (lane < 2) store_at(smem_of_rank(&sm.gave_up, lane), 1);
  };
  // Step kb of a tile to stage st, by one thread.
  const auto load_stage = [&](const Tile& tl, int kb, int st) {
    const int bn_own = p.bn / 2;
    const int m0 = tl.m * kRows + rank * kBM, n0 = tl.n * p.bn + rank * bn_own;
    const uint32_t bar = smem_of_rank(&sm.full[st], 0);
    uint8_t *a = sm.ring + st * stage_bytes, *b = a + kABytes;
    if (rank == 0) mbar_arrive_expect_tx(&sm.full[st], 2 * stage_bytes);
    if (kForm == kGated) {
      tma_load_2d_pair(a, &maps.a[0], bar, kb * kBK, m0);
      tma_load_2d_pair(b, &maps.b[rank], bar, kb * kBK, tl.n * bn_own);
    } else if (kForm == kCols) {
      tma_load_2d_pair(a, &maps.a[0], bar, kb * kBK, m0);
      tma_load_2d_pair(b, &maps.b[0], bar, kb * kBK, n0);
    } else if (kForm == kColsTurned) {
      const int run = kb >= p.first_kblocks, k0 = (kb - run * p.first_kblocks) * kBK;
      for (int i = 0; i < 2; ++i) tma_load_2d_pair(a + i * kBoxBytes, &maps.a[run], bar, m0 + 64 * i, k0);
      tma_load_2d_pair(b, &maps.b[run], bar, k0, n0);
    } else {
      const int second = tl.m >= p.first_tiles, r0 = m0 - second * p.first_tiles * kRows;
      for (int i = 0; i < 2; ++i) tma_load_2d_pair(a + i * kBoxBytes, &maps.a[second], bar, r0 + 64 * i, kb * kBK);
      tma_load_2d_pair(b, &maps.b[0], bar, kb * kBK, n0);
    }
  };
  if (warp == 0) {
    // ================================================================ TMA producer
    Ring ring;
    int fill = 0;
    bool ok = true, ready = true;
    for (int t = worker; ok && t < tiles; t += workers) {
      const Tile tl = tile_of(p, t);
      for (int kb = 0; kb < p.kblocks; ++kb, ++fill) {
        const int st = ring.stage;
        if (!warp_wait_if(ready, &sm.empty[st], ring.round ^ 1, abort, p.err, p.wait_ns)) {
          ok = false;
          break;
        }
        ring.next(stages);
        ready = fill + 1 < stages || mbar_test(&sm.empty[ring.stage], ring.round ^ 1);
        if (lane == 0) load_stage(tl, kb, st);
      }
    }
    launch_dependents();
    // Teardown: every copy issued lands before the block exits. The copies complete on the
    // leader's barriers, so each CTA waits for the MMAs that read its stages, and where
    // something has given up both settle their accounts behind the roles.
    bool landed = ok;
    for (int s = 0; s < stages; ++s) {
      const int n_s = fill > s ? (fill - s + stages - 1) / stages : 0;
      if (n_s && landed) landed = warp_wait(&sm.empty[s], (n_s - 1) & 1, abort, p.err, p.wait_ns);
    }
    if (lane < 2) store_at(smem_of_rank(&sm.loads[rank], lane), fill);  // here and in the other CTA
    if (!landed) give_up();
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ================================================================ MMA issuer
    // A step of 16 in K: 32 bytes of each row (K-major), or 16 rows of 128 bytes (MN-major).
    constexpr uint32_t a_step = a_mn ? 128 : 2, b_step = 2;
    const uint32_t idesc = idesc_bf16_f32(kRows, p.bn, a_mn, false);
    const uint64_t a_desc0 = sdesc_sw128(smem_u32(sm.ring), a_mn ? kBoxBytes : 16, 1024);
    const uint64_t b_desc0 = sdesc_sw128(smem_u32(sm.ring + kABytes), 16, 1024);
    Ring ring;
    int fill = 0, tile = 0;
    bool ok = true, ready = false;
    for (int t = worker; ok && t < tiles; t += workers, ++tile) {
      const int acc = tile & 1;
      // The accumulator's previous tile (tile - 2) must have been read out.
      if (tile >= 2 && !warp_wait(&sm.acc_empty[acc], ((tile >> 1) - 1) & 1, abort, p.err, p.wait_ns)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t d_tmem = tmem + acc * kMaxBN;
      for (int kb = 0; kb < p.kblocks; ++kb, ++fill) {
        const int st = ring.stage;
        if (!warp_wait_if(ready, &sm.full[st], ring.round, abort, p.err, p.wait_ns)) {
          ok = false;
          break;
        }
        ring.next(stages);
        ready = mbar_test(&sm.full[ring.stage], ring.round);
        tc_fence_after();
        const uint32_t at = static_cast<uint32_t>(st) * (stage_bytes >> 4);
        const uint64_t a_desc = a_desc0 + at, b_desc = b_desc0 + at;
#pragma unroll
        for (int kk = 0; kk < kBK / 16; ++kk)
          mma_ss_pair_elect(d_tmem, a_desc + kk * a_step, b_desc + kk * b_step, idesc, (kb > 0 || kk > 0) ? 1u : 0u);
        mma_commit_pair_elect(&sm.empty[st]);
      }
      if (!ok) break;
      mma_commit_pair_elect(&sm.acc_full[acc]);
    }
    // In this CTA alone: the other one does not wait for it, and may be gone when it arrives.
    mma_commit_leader_elect(&sm.done);
    mbar_drain(&sm.done, 0);
    if (!ok) give_up();
    if (lane < 2) {
      store_at(smem_of_rank(&sm.mma_steps, lane), fill);
      store_at(smem_of_rank(&sm.mma_tiles, lane), tile);
    }
    __syncwarp();
  } else if (warp >= kEpiWarp0) {
    // ================================================================ epilogue
    // Two warps for each 32 lanes, which take the tile's groups of 64 columns in turn.
    const int qw = warp & 3;                         // TMEM lanes 32 qw .. 32 qw + 31
    const int half = (warp - kEpiWarp0) >> 2;
    const uint32_t lane_base = static_cast<uint32_t>(qw * 32) << 16;
    uint8_t* buf = sm.out[warp - kEpiWarp0];
    const auto release = [&](int acc) {  // every column of the accumulator has been read
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_at(smem_of_rank(&sm.acc_empty[acc], 0));
    };
    const auto free_again = [&] {  // the store before has left the buffer
      if (lane == 0) bulk_wait_read<0>();
      __syncwarp();
    };
    // 16 bytes: columns 8 e .. 8 e + 7 of this lane's row.
    const auto put = [&](int e, float x0, float x1, float x2, float x3, float x4, float x5, float x6, float x7) {
      *reinterpret_cast<uint4*>(buf + lane * 128 + ((e ^ (lane & 7)) << 4)) =
          make_uint4(pack_bf16x2(x0, x1), pack_bf16x2(x2, x3), pack_bf16x2(x4, x5), pack_bf16x2(x6, x7));
    };
    const auto send = [&](const CUtensorMap* map, int c0, int c1) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (c0 < p.cols && c1 < p.n) tma_store_2d(map, buf, c0, c1);
        bulk_commit();
      }
    };
    int tile = 0;
    bool ok = true;
    for (int t = worker; t < tiles; t += workers, ++tile) {
      const Tile tl = tile_of(p, t);
      const int acc = tile & 1;
      const int m0 = tl.m * kRows + rank * kBM + qw * 32;  // of this warp's lanes
      const int groups = (kForm == kGated ? p.bn / 2 : p.bn) / 64;
      // cols: eight columns a lane, their biases, and the residuals of the next 32 rows, on their way
      // while these are computed (loaded where they are added each waits for memory by itself: 2224 rows of
      // 32 x 8192 took 74 us, not 38).
      const int col = m0 + 8 * (lane & 3);
      const bool on = col < p.cols;  // (a multiple of 8)
      float bias[8] = {};
      uint4 ahead[4] = {};
      const auto fetch_residual = [&](int row0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t row = static_cast<int64_t>(row0) + 8 * k + (lane >> 2);
          if (row < p.n && on) ahead[k] = load8_raw(p.residual + row * p.s_residual + col, p.wide);
        }
      };
      if ((kForm == kCols || kForm == kColsTurned) && half < groups) {
        if (p.residual) fetch_residual(tl.n * p.bn + 64 * half);
        if (kForm == kCols && p.bias && on) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            bias[k] = p.bias_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.bias)[col + k])
                                  : static_cast<const float*>(p.bias)[col + k];
        }
      }
      if (!warp_wait(&sm.acc_full[acc], (tile >> 1) & 1, abort, p.err, p.wait_ns)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t base = tmem + lane_base + acc * kMaxBN;
      if (half >= groups) release(acc);
#pragma unroll 1
      for (int g = half; g < groups; g += 2) {
        const bool last = g + 2 >= groups;
        if (kForm == kGated) {
          const int col0 = tl.n * (p.bn / 2) + 64 * g;
          free_again();
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            uint32_t x[32], y[32];
            tmem_ld32(base + 64 * g + 32 * c, x);
            tmem_ld32(base + p.bn / 2 + 64 * g + 32 * c, y);
            tmem_wait_ld(x);
            tmem_wait_ld(y);
            if (last && c == 1 && !p.keep) release(acc);
            float h[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) h[e] = activate(p.act, __uint_as_float(x[e])) * __uint_as_float(y[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              put(4 * c + e, h[8 * e], h[8 * e + 1], h[8 * e + 2], h[8 * e + 3], h[8 * e + 4], h[8 * e + 5], h[8 * e + 6], h[8 * e + 7]);
          }
          send(&maps.out[0], col0, m0);
          if (!p.keep) continue;
#pragma unroll 1
          for (int k = 0; k < 2; ++k) {
            free_again();
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
              uint32_t x[32];
              tmem_ld32(base + k * (p.bn / 2) + 64 * g + 32 * c, x);
              tmem_wait_ld(x);
              if (last && k == 1 && c == 1) release(acc);
              const auto f = [&](int e) { return __uint_as_float(x[e]); };
#pragma unroll
              for (int e = 0; e < 4; ++e)
                put(4 * c + e, f(8 * e), f(8 * e + 1), f(8 * e + 2), f(8 * e + 3), f(8 * e + 4), f(8 * e + 5), f(8 * e + 6), f(8 * e + 7));
            }
            send(&maps.out[1 + k], col0, m0);
          }
        } else if (kForm == kRowsForm) {
          const int second = tl.m >= p.first_tiles, r0 = m0 - second * p.first_tiles * kRows;
          uint32_t x[32], y[32];
          tmem_ld32(base + 64 * g, x);
          tmem_ld32(base + 64 * g + 32, y);
          tmem_wait_ld(x);
          tmem_wait_ld(y);
          if (last) release(acc);
          free_again();
          const auto f = [&](int e) { return __uint_as_float(e < 32 ? x[e & 31] : y[e & 31]); };
#pragma unroll
          for (int e = 0; e < 8; ++e)
            put(e, f(8 * e), f(8 * e + 1), f(8 * e + 2), f(8 * e + 3), f(8 * e + 4), f(8 * e + 5), f(8 * e + 6), f(8 * e + 7));
          send(&maps.out[second], tl.n * p.bn + 64 * g, r0);
        } else {
          // 32 rows of the result at a time, of which the lanes hold a column each, turned in shared
          // memory: eight columns a lane of every eighth row (16-byte pieces swapped by the row, so
          // that neither side meets a bank twice).
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            const int row0 = tl.n * p.bn + 64 * g + 32 * c;
            uint4 extra[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) extra[k] = ahead[k];
            if (p.residual && (c == 0 || !last)) fetch_residual(row0 + (c == 0 ? 32 : 96));
            uint32_t x[32];
            tmem_ld32(base + 64 * g + 32 * c, x);
            tmem_wait_ld(x);
            if (last && c == 1) release(acc);
#pragma unroll
            for (int e = 0; e < 32; ++e) *reinterpret_cast<uint32_t*>(buf + e * 128 + ((lane * 4) ^ ((e & 7) << 4))) = x[e];
            __syncwarp();
#pragma unroll 1
            for (int pass = 0; pass < 4; ++pass) {
              const int e = 8 * pass + (lane >> 2);
              const int64_t row = row0 + e;
              const uint4 mine = extra[0];
#pragma unroll
              for (int k = 0; k < 3; ++k) extra[k] = extra[k + 1];
              if (row >= p.n || !on) continue;
              const int piece = 2 * (lane & 3), swap = e & 7;
              const float4 lo = *reinterpret_cast<const float4*>(buf + e * 128 + ((piece ^ swap) << 4));
              const float4 hi = *reinterpret_cast<const float4*>(buf + e * 128 + (((piece + 1) ^ swap) << 4));
              float z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, add[8];
              unpack8(mine, add);
              if (kForm == kCols) {
#pragma unroll
                for (int k = 0; k < 8; ++k) z[k] += bias[k];
                if (p.pre) store8(p.pre + row * p.s_pre + col, p.wide, z);
                if (p.act != DLM_ACT_NONE) {
#pragma unroll
                  for (int k = 0; k < 8; ++k) z[k] = activate(p.act, z[k]);
                }
              }
#pragma unroll
              for (int k = 0; k < 8; ++k) z[k] += add[k];
              store8(p.out + row * p.s_out + col, p.wide, z);
            }
            __syncwarp();
          }
        }
      }
    }
    if (!ok) give_up();
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  cg::this_cluster().sync();  // neither CTA's memory goes while the pair's copies and MMAs may use it
  if (sm.gave_up) {           // (the same in both)
    if (threadIdx.x == 0) {
      // The commits that arrive here, one of a barrier on its way at most: the next one needs
      // what has waited for it.
      const int steps = sm.mma_steps, done = sm.mma_tiles;
      bool came = true;
      for (int s = 0; s < stages; ++s) {
        const int n_s = steps > s ? (steps - s + stages - 1) / stages : 0;
        if (n_s && came) came = mbar_drain(&sm.empty[s], (n_s - 1) & 1);
      }
      for (int i = 0; i < 2; ++i) {
        const int n_i = done > i ? (done - i + 1) / 2 : 0;
        if (n_i && came) came = mbar_drain(&sm.acc_full[i], (n_i - 1) & 1);
      }
      // The CTA behind loads what the other one has loaded (into stages that are free, or the
      // other one's would not have been), so that every step's barrier in the leader gets
      // all its bytes; there their number is waited for.
      const int mine = sm.loads[rank], both = max(sm.loads[0], sm.loads[1]);
      int at = 0;
      for (int t = worker; at < both && t < tiles; t += workers) {
        const Tile tl = tile_of(p, t);
        for (int kb = 0; at < both && kb < p.kblocks; ++kb, ++at)
          if (at >= mine) load_stage(tl, kb, at % stages);
      }
      if (rank == 0)
        for (int s = 0; s < stages; ++s) {
          const int n_s = both > s ? (both - s + stages - 1) / stages : 0;
          if (n_s && came) came = mbar_drain(&sm.full[s], (n_s - 1) & 1);
        }
    }
    __syncwarp();
    cg::this_cluster().sync();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------- gradients' element-wise parts

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ uint4 row8(const __nv_bfloat16* base, int64_t row, int64_t stride, int64_t vec) {
  return *reinterpret_cast<const uint4*>(base + row * stride + 8 * vec);
}

// kGate: dg = dout u act'(g), du = dout act(g); else dg = dout act'(g). Rounded to bf16 for the tensor
// cores: each term of the gradients is off by at most 2^-8 relative, as the results are by their own
// rounding. Two vectors a thread in flight. HBM bounds it: 16384 x 8192 with a gate 207 us (1.34 GB,
// 6.5 TB/s, 95 % of a copy), without one 123 (805 MB).
constexpr int kPartThreads = 256;
template <bool kGate>
__global__ void __launch_bounds__(kPartThreads)
    parts_kernel(const __nv_bfloat16* dout, const __nv_bfloat16* gate, const __nv_bfloat16* up, int64_t s_dout, int64_t s_gate,
                 int64_t s_up, int act, int64_t rows, int vecs, uint4* dgate, uint4* dup) {
  constexpr int kLoads = kGate ? 2 : 3;
  wait_for_previous();
  launch_dependents();
  // Row and place in it go on by steps, without a division for each vector.
  const int64_t total = rows * vecs, step = static_cast<int64_t>(gridDim.x) * kPartThreads;
  const unsigned start = blockIdx.x * kPartThreads + threadIdx.x, step_r = gridDim.x * kPartThreads / static_cast<unsigned>(vecs);
  const int step_c = static_cast<int>(gridDim.x * kPartThreads - step_r * vecs);
  int64_t r = start / static_cast<unsigned>(vecs);
  int c = static_cast<int>(start % static_cast<unsigned>(vecs));
  for (int64_t i0 = start; i0 < total; i0 += kLoads * step) {
    uint4 v[kLoads][kGate ? 3 : 2] = {};
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      if (i0 + k * step < total) {
        v[k][0] = row8(dout, r, s_dout, c);
        v[k][1] = row8(gate, r, s_gate, c);
        if constexpr (kGate) v[k][2] = row8(up, r, s_up, c);
      }
      r += step_r;
      c += step_c;
      if (c >= vecs) {
        c -= vecs;
        ++r;
      }
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int64_t i = i0 + k * step;
      if (i >= total) continue;
      float d[8], g[8], u[8];
      unpack8(v[k][0], d);
      unpack8(v[k][1], g);
      if constexpr (kGate) unpack8(v[k][2], u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float value, slope;
        activate_grad(act, g[e], &value, &slope);
        if constexpr (kGate) {
          g[e] = d[e] * u[e] * slope;
          u[e] = d[e] * value;
        } else {
          g[e] = d[e] * slope;
        }
      }
      dgate[i] = pack8(g);
      if constexpr (kGate) dup[i] = pack8(u);
    }
  }
}

// dz = dout act'(pre) (not written without an activation), and the sums of its columns: 8 kLanes
// columns a CTA, 256 / kLanes rows at a time, four of them a thread in flight. The CTAs of a cluster
// share a run of rows, whose sums its first one adds up in their order: to `sums`, or, where there is one
// run, to `dbias`.
template <int kLanes>
__global__ void __launch_bounds__(kPartThreads, 4)
    bias_parts_kernel(const __nv_bfloat16* dout, const __nv_bfloat16* pre, int64_t s_dout, int64_t s_pre, int act, int64_t rows,
                      int64_t rows_per_cta, int vecs, uint4* dz, float* sums, void* dbias, int bias_bf16) {
  constexpr int kLoads = 4, kRowsOnce = kPartThreads / kLanes, kCols = 8 * kLanes;
  __shared__ float part[kRowsOnce][kCols + 1], total[kCols];
  wait_for_previous();
  launch_dependents();
  const int lane = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
  const int ranks = static_cast<int>(cg::this_cluster().num_blocks()), rank = static_cast<int>(cg::this_cluster().block_rank());
  const int64_t strip = blockIdx.x / ranks, c = strip * kLanes + lane, run = static_cast<int64_t>(blockIdx.y) * ranks + rank;
  const int64_t r0 = run * rows_per_cta, r1 = r0 + rows_per_cta < rows ? r0 + rows_per_cta : rows;
  float sum[8] = {};
  for (int64_t r = r0 + row; r < r1 && c < vecs; r += kLoads * kRowsOnce) {
    uint4 d4[kLoads] = {}, z4[kLoads] = {};
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (r + k * kRowsOnce < r1) {
        d4[k] = row8(dout, r + k * kRowsOnce, s_dout, c);
        if (pre) z4[k] = row8(pre, r + k * kRowsOnce, s_pre, c);
      }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      if (r + k * kRowsOnce >= r1) continue;
      float d[8];
      unpack8(d4[k], d);
      if (pre) {
        float z[8];
        unpack8(z4[k], z);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float value, slope;
          activate_grad(act, z[e], &value, &slope);
          d[e] *= slope;
        }
        dz[(r + k * kRowsOnce) * vecs + c] = pack8(d);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += d[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[row][8 * lane + e] = sum[e];
  __syncthreads();
  if (threadIdx.x < kCols) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kRowsOnce; ++i) s += part[i][threadIdx.x];
    total[threadIdx.x] = s;
  }
  cg::this_cluster().sync();
  const int64_t cols = static_cast<int64_t>(vecs) * 8, col = strip * kCols + threadIdx.x;
  if (rank == 0 && threadIdx.x < kCols && col < cols) {
    float s = 0.f;
    for (int i = 0; i < ranks; ++i) s += *cg::this_cluster().map_shared_rank(total + threadIdx.x, i);
    if (sums)
      sums[blockIdx.y * cols + col] = s;
    else if (bias_bf16)
      static_cast<__nv_bfloat16*>(dbias)[col] = __float2bfloat16_rn(s);
    else
      static_cast<float*>(dbias)[col] = s;
  }
  cg::this_cluster().sync();  // nobody's sums go while the first one reads them
}

// The sums of all runs, a thread a column.
__global__ void __launch_bounds__(kPartThreads) bias_sum_kernel(const float* sums, int parts, int cols, void* out, int bf16) {
  wait_for_previous();
  launch_dependents();
  const int col = blockIdx.x * kPartThreads + threadIdx.x;
  if (col >= cols) return;
  float s = 0.f;
#pragma unroll 8
  for (int i = 0; i < parts; ++i) s += sums[static_cast<int64_t>(i) * cols + col];
  if (bf16)
    static_cast<__nv_bfloat16*>(out)[col] = __float2bfloat16_rn(s);
  else
    static_cast<float*>(out)[col] = s;
}

// x [rows, cols] transposed, [cols, pad]: 64 x 64 a CTA (what lies behind the last row is left
// as it is: the map of the result ends there). HBM bounds it: 16384 x 2048 21 us (134 MB, 6.3 TB/s).
__global__ void __launch_bounds__(kPartThreads)
    transpose_kernel(const __nv_bfloat16* x, int64_t stride, int64_t rows, int cols, int64_t pad, uint4* out) {
  __shared__ uint32_t tile[64][33];  // rows of 32 pairs of columns
  wait_for_previous();
  launch_dependents();
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * 64;
  const int d0 = blockIdx.y * 64, r = threadIdx.x >> 3, v = threadIdx.x & 7;
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (r0 + r + i < rows && d0 + 8 * v < cols) u = row8(x + d0, r0 + r + i, stride, v);
    tile[r + i][4 * v] = u.x;
    tile[r + i][4 * v + 1] = u.y;
    tile[r + i][4 * v + 2] = u.z;
    tile[r + i][4 * v + 3] = u.w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int c = r + i, shift = (c & 1) * 16;
    if (d0 + c >= cols) continue;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k] = (tile[8 * v + 2 * k][c >> 1] >> shift & 0xFFFFu) | (tile[8 * v + 2 * k + 1][c >> 1] >> shift) << 16;
    out[((d0 + c) * pad + r0) / 8 + v] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---------------------------------------------------------------- host side

int sm_count() {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool aligned(const void* p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0; }

template <int kForm>
int pairs_of() {
  const auto kernel = product_kernel<kForm>;
  if (allow_smem(reinterpret_cast<const void*>(kernel), static_cast<int>(kSmemBytes)) != cudaSuccess) return 0;
  return active_clusters(reinterpret_cast<const void*>(kernel), 2, kThreads, kSmemBytes);
}

template <int kForm>
int launch_product(const Maps& m, Params p, int workers, cudaStream_t stream) {
  p.err = device_error_word();
  p.wait_ns = wait_budget_ns();
  const int64_t tiles = static_cast<int64_t>(p.row_tiles) * p.col_tiles;
  if (workers < 1) return fail(DLM_ERR_CUDA, "product launch: no place for a pair of CTAs");
  const int64_t run = tiles < workers ? tiles : workers;
  const cudaError_t e = launch_overlapped(product_kernel<kForm>, dim3(static_cast<unsigned>(2 * run)), kThreads, kSmemBytes, stream, 2,
                                          true, m, p);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "product launch: %s", cudaGetErrorString(e));
}

int launched(cudaError_t e, const char* what) {
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
}

// A matrix as the tensor maps take it.
int operand_map(CUtensorMap* map, const Matrix& x, int box_rows) {
  return make_matrix_map(map, x.data, true, x.rows, x.cols, x.stride, box_rows);
}

// out = act(x w^T + bias) + residual (turned: w's columns instead of its rows; two runs of K).
int launch_cols(const Matrix* x, const Matrix* w, int runs, bool turned, const Epilogue& ep, cudaStream_t stream) {
  const int64_t N = x[0].rows, M = turned ? w[0].cols : w[0].rows;
  const int64_t kblocks = ceil_div(x[0].cols, kBK);
  const int workers = turned ? pairs_of<kColsTurned>() : pairs_of<kCols>();
  const ProductPlan plan = plan_cols(N, M, runs * kblocks, turned, workers);
  if (!plan.pairs) return launch_few_cols(x, w, runs, turned, ep, plan.few, stream);
  Params p = {};
  p.row_tiles = static_cast<int>(ceil_div(M, kRows));
  p.bn = plan.bn;
  p.col_tiles = static_cast<int>(ceil_div(N, p.bn));
  Maps m = {};
  int st;
  for (int i = 0; i < runs; ++i) {
    if ((st = operand_map(&m.a[i], w[i], turned ? 64 : kBM)) != DLM_OK) return st;
    if ((st = operand_map(&m.b[i], x[i], p.bn / 2)) != DLM_OK) return st;
  }
  p.first_kblocks = static_cast<int>(kblocks);
  p.kblocks = runs * p.first_kblocks;
  p.act = ep.act;
  p.n = static_cast<int>(N);
  p.cols = static_cast<int>(M);
  p.bias = ep.bias;
  p.bias_bf16 = ep.bias_bf16;
  p.residual = static_cast<const __nv_bfloat16*>(ep.residual);
  p.out = static_cast<__nv_bfloat16*>(ep.out);
  p.pre = static_cast<__nv_bfloat16*>(ep.pre);
  p.s_residual = ep.s_residual;
  p.s_out = ep.s_out;
  p.s_pre = ep.s_pre;
  p.wide = aligned(ep.out, ep.s_out) && (!ep.residual || aligned(ep.residual, ep.s_residual)) && (!ep.pre || aligned(ep.pre, ep.s_pre));
  return turned ? launch_product<kColsTurned>(m, p, workers, stream) : launch_product<kCols>(m, p, workers, stream);
}

size_t take(size_t* at, size_t bytes) {
  const size_t here = *at;
  *at += (bytes + 255) / 256 * 256;
  return here;
}

int64_t pad_rows(int64_t n) { return ceil_div(n, 64) * 64; }

struct GradLayout {
  size_t dz, second, turned, sums, bytes;
};
GradLayout grad_layout(int64_t N, int64_t m, int64_t d, int matrices) {
  GradLayout l = {};
  l.dz = take(&l.bytes, static_cast<size_t>(N) * m * 2);
  if (matrices == 2) l.second = take(&l.bytes, static_cast<size_t>(N) * m * 2);
  l.turned = take(&l.bytes, static_cast<size_t>(d) * pad_rows(N) * 2);
  if (matrices == 1) l.sums = take(&l.bytes, static_cast<size_t>(bias_split(N, m).runs) * m * 4);
  return l;
}

// dgate and dup, or (kGate false, g the projection's pre) dgate alone.
template <bool kGate>
int launch_parts(const Matrix& dout, const Matrix& g, const Matrix& up, int act, void* dgate, void* dup, cudaStream_t stream) {
  const int64_t ctas = ceil_div(g.rows * (g.cols / 8), kPartThreads), most = static_cast<int64_t>(sm_count()) * 8;
  return launched(launch_overlapped(parts_kernel<kGate>, dim3(static_cast<unsigned>(ctas < most ? ctas : most)), kPartThreads, 0, stream, 1,
                                    true, static_cast<const __nv_bfloat16*>(dout.data), static_cast<const __nv_bfloat16*>(g.data),
                                    static_cast<const __nv_bfloat16*>(up.data), dout.stride, g.stride, up.stride, act, g.rows,
                                    static_cast<int>(g.cols / 8), static_cast<uint4*>(dgate), static_cast<uint4*>(dup)),
                  "gradient parts");
}

int launch_transpose(const Matrix& x, void* out, Matrix* turned, cudaStream_t stream) {
  *turned = {out, x.cols, x.rows, pad_rows(x.rows)};
  const dim3 grid(static_cast<unsigned>(pad_rows(x.rows) / 64), static_cast<unsigned>(ceil_div(x.cols, 64)));
  return launched(launch_overlapped(transpose_kernel, grid, kPartThreads, 0, stream, 1, true, static_cast<const __nv_bfloat16*>(x.data),
                                    x.stride, x.rows, static_cast<int>(x.cols), turned->stride, static_cast<uint4*>(out)),
                  "transposition");
}

// out[i] = z[i]^T x for `count` matrices z of the same shape; turned: room for x transposed.
int launch_rows(const Matrix* z, const Matrix& x, void* turned, const Matrix* out, int count, cudaStream_t stream) {
  const int workers = pairs_of<kRowsForm>();
  const int64_t row_tiles = count * ceil_div(z[0].cols, kRows), kblocks = ceil_div(x.rows, kBK);
  const ProductPlan plan = plan_rows(z[0].cols, x.cols, kblocks, count, workers);
  if (!plan.pairs) return launch_few_outer(z, x, out, count, plan.few, stream);
  Matrix xt;
  int st;
  if ((st = launch_transpose(x, turned, &xt, stream)) != DLM_OK) return st;
  Params p = {};
  p.first_tiles = static_cast<int>(ceil_div(z[0].cols, kRows));
  p.row_tiles = static_cast<int>(row_tiles);
  p.bn = plan.bn;
  p.col_tiles = static_cast<int>(ceil_div(xt.rows, p.bn));
  p.kblocks = p.first_kblocks = static_cast<int>(kblocks);
  p.n = static_cast<int>(z[0].cols);
  p.cols = static_cast<int>(xt.rows);
  Maps m = {};
  for (int i = 0; i < count; ++i) {
    if ((st = operand_map(&m.a[i], z[i], 64)) != DLM_OK) return st;
    if ((st = operand_map(&m.out[i], out[i], 32)) != DLM_OK) return st;
  }
  if ((st = operand_map(&m.b[0], xt, p.bn / 2)) != DLM_OK) return st;
  return launch_product<kRowsForm>(m, p, workers, stream);
}

// dx = sum z[i] w[i] + what ep adds (none without ep.out), dw[i] = z[i]^T x (none without data).
int launch_gradients(const Matrix* z, const Matrix* w, int count, const Epilogue& ep, const Matrix& x, void* turned, const Matrix* dw,
                     cudaStream_t stream) {
  const GradientsPlan plan = plan_gradients(x.rows, z[0].cols, x.cols, count, pairs_of<kColsTurned>(), pairs_of<kRowsForm>());
  if (plan.together) {
    if (ep.out && dw[0].data) return launch_few_gradients(z, w, count, ep, plan.x.few, x, dw, plan.w.few, stream);
    return ep.out ? launch_few_cols(z, w, count, true, ep, plan.x.few, stream)
                  : dw[0].data ? launch_few_outer(z, x, dw, count, plan.w.few, stream) : DLM_OK;
  }
  int st;
  if (ep.out && (st = launch_cols(z, w, count, true, ep, stream)) != DLM_OK) return st;
  return dw[0].data ? launch_rows(z, x, turned, dw, count, stream) : DLM_OK;
}

}  // namespace

// ---------------------------------------------------------------- which form a call takes

namespace {

// Columns of a tile and the time as fitted to measurements (us): 256, or 128 where those leave pairs
// without a tile or much of the last one empty. A K step takes 0.27 to 0.29 us, 0.205 of 128 columns
// (0.245 with an MN-major A), a tile no less than its epilogue, which the last one adds: those that are
// turned in shared memory take longer.
struct PairPlan {
  int bn;
  double us;
};
constexpr double kTurnUs = 3.0;  // the launch that transposes x for the weights' gradients
PairPlan plan_pairs(Form form, int64_t cols, int64_t row_tiles, int64_t kblocks, int workers) {
  const bool a_mn = form == kColsTurned || form == kRowsForm, turned = form == kCols || form == kColsTurned;
  PairPlan best = {256, 1e300};
  for (int bn = 256; bn >= 128 && workers > 0; bn /= 2) {
    const double rounds = static_cast<double>(ceil_div(ceil_div(cols, bn) * row_tiles, workers));
    const double step = bn == 256 ? 0.28 : a_mn ? 0.245 : 0.205, k = static_cast<double>(kblocks) * step;
    const double epilogue = bn == 256 ? (turned ? 4.0 : 2.4) : (turned ? 2.4 : 1.5);
    const double us = 3.2 + rounds * (k > epilogue ? k : epilogue) + epilogue;
    if (us < best.us - 1e-9) best = {bn, us};
  }
  return best;
}

ProductPlan faster(const PairPlan& pairs, double extra, const FewPlan& few) {
  const bool some = few.us < pairs.us + extra;
  return {!some, pairs.bn, few, some ? few.us : pairs.us + extra};
}

}  // namespace

ProductPairs product_pairs() { return {pairs_of<kGated>(), pairs_of<kCols>(), pairs_of<kColsTurned>(), pairs_of<kRowsForm>()}; }

ProductPlan plan_gated(int64_t N, int64_t f, int64_t kblocks, int workers) {
  return faster(plan_pairs(kGated, 2 * f, ceil_div(N, kRows), kblocks, workers), 0.0, plan_few(N, ceil_div(f, 64), kblocks, 1, false));
}

ProductPlan plan_cols(int64_t N, int64_t M, int64_t kblocks, bool turned, int workers) {
  return faster(plan_pairs(turned ? kColsTurned : kCols, N, ceil_div(M, kRows), kblocks, workers), 0.0,
                plan_few(N, ceil_div(M, kBM), kblocks, 1, false));
}

ProductPlan plan_rows(int64_t M, int64_t d, int64_t kblocks, int count, int workers) {
  return faster(plan_pairs(kRowsForm, d, count * ceil_div(M, kRows), kblocks, workers), kTurnUs,
                plan_few(M, ceil_div(d, kBM), kblocks, count, true));
}

GradientsPlan plan_gradients(int64_t N, int64_t m, int64_t d, int count, int x_workers, int w_workers) {
  const int64_t x_tiles = ceil_div(d, kBM), x_kblocks = count * ceil_div(m, kBK), w_kblocks = ceil_div(N, kBK);
  // In one launch, or apart, whichever is fitted as faster, by the sizes alone, so that each has the
  // same bits without the other. In one launch the longer one takes its time and the shorter one a
  // tenth of its own, where all CTAs run at once, two an SM (64 x 2048 x 8192 with a gate: 43.2 -> 35.5 us
  // with 128 CTAs for dx; 256 x 2048 x 8192: 64.7 -> 48.1 with 128, 65.5 with 256). CTAs that read cost
  // those that write a little each.
  GradientsPlan plan = {};
  FewPlan fx = {}, fw = {};
  double both = 1e300;
  for (int s = 1; s <= 8; s *= 2) {
    const FewPlan a = plan_few(N, x_tiles, x_kblocks, 1, false, s), b = plan_few(m, x_tiles, w_kblocks, count, true, s, true);
    const int64_t x_ctas = x_tiles * ceil_div(N, a.n) * s;
    if (x_ctas + few_outer_ctas(m, x_tiles, count, b) > 2 * 152) continue;
    const double us = (a.us > b.us ? a.us + 0.1 * b.us : b.us + 0.1 * a.us) + 0.01 * static_cast<double>(x_ctas);
    if (us >= both) continue;
    both = us;
    fx = a;
    fw = b;
  }
  plan.x = plan_cols(N, d, x_kblocks, true, x_workers);
  plan.w = plan_rows(m, d, w_kblocks, count, w_workers);
  plan.together = both < plan.x.us + plan.w.us + 3.0;
  if (plan.together) {
    plan.x = {false, 0, fx, fx.us};
    plan.w = {false, 0, fw, fw.us};
  }
  return plan;
}

// How the sums of dz's columns are split: strips of 8 `lanes` columns; runs of rows, whose sums are kept
// (one run needs no second launch); CTAs of a cluster that share a run. As many CTAs as run at once,
// four an SM, with 64 rows each or more: with twice as many 16384 x 8192 took 159 us. Pieces of 512
// bytes of a row instead of 128 pay where there is much to read, with clusters only to keep the runs few
// (16384 x 8192: 132 us, 805 MB at 6.1 TB/s, against 152; 2048 x 2048: 9.8 against 8.4).
BiasSplit bias_split(int64_t N, int64_t m) {
  constexpr int64_t kCtas = 4 * 152, kMuch = 2048, kManyRuns = 64;  // (608 CTAs in clusters of eight: 76 runs at most)
  const int64_t most = ceil_div(N, 64);
  int ranks = 1;
  if (ceil_div(m, 256) * most >= kMuch) {
    int64_t all = kCtas / ceil_div(m, 256);
    all = all < 1 ? 1 : all < most ? all : most;
    while (ranks < 8 && all / ranks > kManyRuns) ranks *= 2;
    return {32, all / ranks, ranks};
  }
  const int64_t want = ceil_div(kCtas, ceil_div(m, 64)), all = want < most ? want : most;
  while (ranks < 8 && ranks * 2 <= all) ranks *= 2;
  return {8, all > 64 ? ceil_div(all, ranks) : 1, ranks};
}

int launch_gated(const GatedArgs& a, cudaStream_t stream) {
  const int64_t f = a.w_gate.rows, row_tiles = ceil_div(a.x.rows, kRows), kblocks = ceil_div(a.x.cols, kBK);
  const int workers = pairs_of<kGated>();
  const ProductPlan plan = plan_gated(a.x.rows, f, kblocks, workers);
  if (!plan.pairs) return launch_few_gated(a, plan.few, stream);
  Params p = {};
  p.row_tiles = static_cast<int>(row_tiles);
  p.bn = plan.bn;
  p.col_tiles = static_cast<int>(ceil_div(f, p.bn / 2));
  p.kblocks = p.first_kblocks = static_cast<int>(kblocks);
  p.act = a.act;
  p.n = static_cast<int>(a.x.rows);
  p.cols = static_cast<int>(a.w_gate.rows);
  p.keep = a.gate.data != nullptr;
  Maps m = {};
  int st;
  if ((st = operand_map(&m.a[0], a.x, kBM)) != DLM_OK) return st;
  if ((st = operand_map(&m.b[0], a.w_gate, p.bn / 2)) != DLM_OK) return st;
  if ((st = operand_map(&m.b[1], a.w_up, p.bn / 2)) != DLM_OK) return st;
  if ((st = operand_map(&m.out[0], a.out, 32)) != DLM_OK) return st;
  if (p.keep && (st = operand_map(&m.out[1], a.gate, 32)) != DLM_OK) return st;
  if (p.keep && (st = operand_map(&m.out[2], a.up, 32)) != DLM_OK) return st;
  return launch_product<kGated>(m, p, workers, stream);
}

size_t gated_grad_workspace_bytes(int64_t N, int64_t f, int64_t d) { return grad_layout(N, f, d, 2).bytes; }

int launch_gated_grad(const GatedArgs& a, cudaStream_t stream) {
  const int64_t N = a.x.rows, f = a.w_gate.rows, d = a.x.cols;
  const GradLayout l = grad_layout(N, f, d, 2);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  const Matrix dz[2] = {{ws + l.dz, N, f, f}, {ws + l.second, N, f, f}}, w[2] = {a.w_gate, a.w_up}, dw[2] = {a.dw_gate, a.dw_up};
  const int st = launch_parts<true>(a.dout, a.gate, a.up, a.act, dz[0].data, dz[1].data, stream);
  if (st != DLM_OK) return st;
  Epilogue ep = {};
  ep.residual = a.add;
  ep.s_residual = a.s_add;
  ep.out = a.dx;
  ep.s_out = a.s_dx;
  return launch_gradients(dz, w, 2, ep, a.x, ws + l.turned, dw, stream);
}

size_t linear_workspace_bytes(int64_t N, int64_t m, int64_t k) {
  (void)N;
  (void)m;
  (void)k;
  return 0;
}

int launch_linear(const LinearArgs& a, cudaStream_t stream) { return launch_cols(&a.x, &a.w, 1, false, a.ep, stream); }

size_t linear_grad_workspace_bytes(int64_t N, int64_t m, int64_t k) { return grad_layout(N, m, k, 1).bytes; }

int launch_linear_grad(const LinearArgs& a, cudaStream_t stream) {
  const int64_t N = a.x.rows, m = a.w.rows, k = a.x.cols;
  const GradLayout l = grad_layout(N, m, k, 1);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  Matrix dz = a.dout;
  int st;
  if (a.pre.data) dz = {ws + l.dz, N, m, m};
  if (a.dbias) {
    const BiasSplit split = bias_split(N, m);
    const int64_t rows = ceil_div(N, split.runs * split.ranks);
    float* sums = split.runs > 1 ? reinterpret_cast<float*>(ws + l.sums) : nullptr;
    const dim3 grid(static_cast<unsigned>(ceil_div(m, 8 * split.lanes) * split.ranks), static_cast<unsigned>(split.runs));
    st = launched(launch_overlapped(split.lanes == 32 ? bias_parts_kernel<32> : bias_parts_kernel<8>, grid, kPartThreads, 0, stream,
                                    split.ranks, true, static_cast<const __nv_bfloat16*>(a.dout.data),
                                    static_cast<const __nv_bfloat16*>(a.pre.data), a.dout.stride, a.pre.stride, a.ep.act, N, rows,
                                    static_cast<int>(m / 8), reinterpret_cast<uint4*>(ws + l.dz), sums, a.dbias, a.ep.bias_bf16),
                  "gradient parts");
    if (st != DLM_OK) return st;
    if (sums) {
      st = launched(launch_overlapped(bias_sum_kernel, dim3(static_cast<unsigned>(ceil_div(m, kPartThreads))), kPartThreads, 0, stream, 1,
                                      true, static_cast<const float*>(sums), static_cast<int>(split.runs), static_cast<int>(m), a.dbias,
                                      a.ep.bias_bf16),
                    "bias gradient");
      if (st != DLM_OK) return st;
    }
  } else if (a.pre.data) {
    if ((st = launch_parts<false>(a.dout, a.pre, Matrix{}, a.ep.act, dz.data, nullptr, stream)) != DLM_OK) return st;
  }
  Epilogue ep = a.ep;  // of d x
  ep.act = DLM_ACT_NONE;
  ep.bias = nullptr;
  return launch_gradients(&dz, &a.w, 1, ep, a.x, ws + l.turned, &a.dw, stream);
}

}  // namespace dlm
