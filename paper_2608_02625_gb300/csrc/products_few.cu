// The products of a feed-forward block (products.cu) where they are small: few rows, as in
// serving, or too few output tiles for pairs of CTAs.
//
// The result is computed transposed, in tiles of 128 of its columns (TMEM lanes) and n of its
// rows, 16 to 128, so that few rows waste little of an MMA and the weights, which bound it,
// stream through at 16 KB a K step. K is split over the CTAs of a cluster, up to 8 of them, for
// enough CTAs to keep HBM busy: each leaves its fp32 sums in its shared memory, and each reads
// its share of the rows from all of them (distributed shared memory, in the order of the ranks: the
// same bits every time) for the epilogue. No partial sums go through memory, and no second launch.
//   gated   A is 64 gate rows and the same 64 up rows; the epilogue has both in shared memory
//   cols    A the weight's rows (K-major), B the rows of x
//   turned  A the weight's columns (MN-major), B the rows of dz; K in up to two runs
//   outer   dW = dz^T x: A the columns of x, B those of dz (both MN-major, as they lie)
// Two CTAs an SM, more where K is short. Where dW's K is not split (few_weights), CTAs take one tile
// after another and write it while the next one is computed.
// HBM bounds it, behind some 3 us of launch, first loads and joins: one row against 33 MB of weights
// (2048 x 8192) takes 8.9 us, 67 MB with a gate 14.8, where 4.9 and 9.9 are what reading them takes.
// Every wait is bounded; on expiry the kernel sets DLM_DEVERR_TIMEOUT, lets what it has on its way
// land and goes on to the cluster's barriers with whatever it has.
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

constexpr int kBM = 128;               // lanes: columns of the result (gated: 64, twice)
constexpr int kBK = 64;                // K of a stage: 128 bytes of bf16
constexpr int kThreads = 256;          // warp 0 TMA, warp 1 MMA; all of them the epilogue
constexpr int kABytes = kBM * kBK * 2;
constexpr int kBoxBytes = 64 * 128;    // an MN-major box: 64 K rows of 64 columns
constexpr int kSms = 152;
constexpr int kClustered = 256;  // CTAs in clusters of four or eight that find room at once, two an SM
constexpr int kMaxStages = 8;
constexpr int kStageRoom = 108 * 1024;  // of a CTA, so that two fit on an SM
constexpr int kAloneRoom = 192 * 1024;  // of a CTA with an SM to itself

enum Form { kGated, kCols, kTurned, kOuter };

struct Bars {
  uint64_t full[kMaxStages];   // stage loaded           (TMA -> MMA)
  uint64_t empty[kMaxStages];  // stage read by its MMAs (MMA -> TMA)
  uint64_t done;               // every MMA completed
  uint64_t acc_full[2];        // few_weights: accumulator complete (MMA -> epilogue)
  uint64_t acc_empty[2];       // accumulator read out              (epilogue -> MMA)
  uint32_t tmem_base;
  int abort;
};

struct Maps {
  CUtensorMap a[2], b[2];  // [1]: up (gated), the second run of K (turned), the second matrix (outer: b)
};

// out[0]: the result; gated: gate and up behind it (may be null); outer: the second matrix's.
struct Params {
  int col_tiles, first_tiles;  // tiles of n rows of the result; outer: those of the first matrix
  int tiles;                   // few_weights: all
  int n;                       // rows of a tile
  int kblocks, first_kblocks;  // K steps; those of the first run
  int splits, stages;
  int rows, cols;              // extents of the result
  int act, bias_bf16;
  int wide;                    // rows of out, pre and residual are 16-byte aligned
  const void* bias;
  const __nv_bfloat16* residual;
  __nv_bfloat16* out[3];
  __nv_bfloat16* pre;
  int64_t s_residual, s_out[3], s_pre;
  uint32_t tmem_cols;
  int* err;
  uint64_t wait_ns;
};

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* err, uint64_t budget_ns) {
  const bool ok = mbar_wait_for<true>(bar, parity, abort, err, budget_ns);
  return __all_sync(0xffffffffu, ok);
}

// The stages in turn. (With fill % stages and fill / stages a step took 600 cycles, whatever it
// loaded: two divisions in a warp of its own.)
struct Ring {
  int stage = 0, round = 0;  // round: the parity of this pass over the stages
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) {
      stage = 0;
      round ^= 1;
    }
  }
};

// A wait that asked before (`ready`, of the same phase): to look at a barrier takes some 170
// cycles, under which the step before is issued.
__device__ __forceinline__ bool warp_wait_if(bool ready, uint64_t* bar, uint32_t parity, volatile int* abort, int* err, uint64_t budget_ns) {
  if (!kCheckBounds && __all_sync(0xffffffffu, ready)) return true;
  return warp_wait(bar, parity, abort, err, budget_ns);
}

__device__ __forceinline__ uint32_t smem_at_rank(uint32_t addr, uint32_t rank) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  return there;
}

__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ float4 load_own(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

template <int kForm>
__device__ __forceinline__ void few_product(const Maps& maps, const Params& p, int block) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Bars bars;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  constexpr bool a_mn = kForm == kTurned || kForm == kOuter, b_mn = kForm == kOuter;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = block % p.splits, tile = block / p.splits;
  const int row_tile = tile / p.col_tiles, col_tile = tile % p.col_tiles;
  const int second = kForm == kOuter && col_tile >= p.first_tiles;
  const int m0 = row_tile * (kForm == kGated ? 64 : kBM);          // first column of the result
  const int n0 = (col_tile - second * p.first_tiles) * p.n;        // first row
  const int k0 = static_cast<int>(static_cast<int64_t>(p.kblocks) * rank / p.splits);
  const int k1 = static_cast<int>(static_cast<int64_t>(p.kblocks) * (rank + 1) / p.splits);
  const int b_bytes = p.n * 128, stage_bytes = kABytes + b_bytes;

  if (threadIdx.x == 32) {
    prefetch_tmap(&maps.a[0]);
    prefetch_tmap(&maps.b[second]);
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&bars.full[s], 1);
      mbar_init(&bars.empty[s], 1);
    }
    mbar_init(&bars.done, 1);
    bars.abort = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    tmem_alloc(&bars.tmem_base, p.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem_base;
  volatile int* abort = &bars.abort;
  wait_for_previous();

  // This CTA's rows of the tile, eight columns a thread, and the residuals of a thread's next rows, on
  // their way from the start.
  const int valid = min(p.n, p.rows - n0);
  const int c0 = static_cast<int>(static_cast<int64_t>(valid) * rank / p.splits);
  const int c1 = static_cast<int>(static_cast<int64_t>(valid) * (rank + 1) / p.splits);
  constexpr int kGroups = kForm == kGated ? 8 : 16;  // of eight columns
  constexpr int kRowsOnce = kThreads / kGroups;
  const int i = 8 * (threadIdx.x % kGroups), col = m0 + i, first = c0 + threadIdx.x / kGroups;
  const bool adds = (kForm == kCols || kForm == kTurned) && p.residual && col < p.cols;  // (a multiple of 8)
  constexpr int kAhead = 2;
  uint4 ahead[kAhead] = {};
  const auto residual_of = [&](int c) {
    return adds && c < c1 ? load8_raw(p.residual + (static_cast<int64_t>(n0) + c) * p.s_residual + col, p.wide) : make_uint4(0, 0, 0, 0);
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k) ahead[k] = residual_of(first + k * kRowsOnce);

  if (warp == 0) {
    // ================================================================ TMA producer
    Ring ring;
    int fill = 0;
    bool ready = true;
    for (int kb = k0; kb < k1; ++kb, ++fill) {
      const int st = ring.stage;
      if (!warp_wait_if(ready, &bars.empty[st], ring.round ^ 1, abort, p.err, p.wait_ns)) break;
      ring.next(p.stages);
      ready = fill + 1 < p.stages || mbar_test(&bars.empty[ring.stage], ring.round ^ 1);
      if (lane == 0) {
        uint8_t *a = smem + st * stage_bytes, *b = a + kABytes;
        uint64_t* bar = &bars.full[st];
        mbar_arrive_expect_tx(bar, stage_bytes);
        if (kForm == kGated) {
          tma_load_2d(a, &maps.a[0], bar, kb * kBK, m0);
          tma_load_2d(a + kABytes / 2, &maps.a[1], bar, kb * kBK, m0);
          tma_load_2d(b, &maps.b[0], bar, kb * kBK, n0);
        } else if (kForm == kCols) {
          tma_load_2d(a, &maps.a[0], bar, kb * kBK, m0);
          tma_load_2d(b, &maps.b[0], bar, kb * kBK, n0);
        } else if (kForm == kTurned) {
          const int run = kb >= p.first_kblocks, k = (kb - run * p.first_kblocks) * kBK;
          for (int i = 0; i < 2; ++i) tma_load_2d(a + i * kBoxBytes, &maps.a[run], bar, m0 + 64 * i, k);
          tma_load_2d(b, &maps.b[run], bar, k, n0);
        } else {
          for (int i = 0; i < 2; ++i) tma_load_2d(a + i * kBoxBytes, &maps.a[0], bar, m0 + 64 * i, kb * kBK);
          for (int i = 0; i < p.n / 64; ++i) tma_load_2d(b + i * kBoxBytes, &maps.b[second], bar, n0 + 64 * i, kb * kBK);
        }
      }
    }
    launch_dependents();
    if (lane == 0)  // every copy issued lands, whoever has given up
      for (int s = 0; s < p.stages; ++s) {
        const int n_s = fill > s ? (fill - s + p.stages - 1) / p.stages : 0;
        if (n_s) mbar_drain(&bars.full[s], (n_s - 1) & 1);
      }
    __syncwarp();
  } else if (warp == 1) {
    // ================================================================ MMA issuer
    constexpr uint32_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;
    const uint32_t idesc = idesc_bf16_f32(kBM, p.n, a_mn, b_mn);
    const uint64_t a_desc0 = sdesc_sw128(smem_u32(smem), a_mn ? kBoxBytes : 16, 1024);
    const uint64_t b_desc0 = sdesc_sw128(smem_u32(smem + kABytes), b_mn ? kBoxBytes : 16, 1024);
    Ring ring;
    int fill = 0;
    bool ready = false;
    for (int kb = k0; kb < k1; ++kb, ++fill) {
      const int st = ring.stage;
      if (!warp_wait_if(ready, &bars.full[st], ring.round, abort, p.err, p.wait_ns)) break;
      ring.next(p.stages);
      ready = mbar_test(&bars.full[ring.stage], ring.round);
      tc_fence_after();
      const uint32_t at = static_cast<uint32_t>(st) * (stage_bytes >> 4);
#pragma unroll
      for (int kk = 0; kk < kBK / 16; ++kk)
        mma_ss_elect(tmem, a_desc0 + at + kk * a_step, b_desc0 + at + kk * b_step, idesc, (fill > 0 || kk > 0) ? 1u : 0u);
      mma_commit_elect(&bars.empty[st]);
    }
    mma_commit_elect(&bars.done);
    mbar_drain(&bars.done, 0);
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();

  // ================================================================ sums to shared memory
  // [row of the tile][lane], over the stages, which nothing uses any more. (Rows are as many as
  // fill a load; what is behind the valid ones is not read.)
  const uint32_t sums = smem_u32(smem);
  for (int c = (warp >> 2) * 32; c < valid; c += 64) {
    uint32_t x[32];
    tmem_ld32(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + c, x);
    tmem_wait_ld(x);
    float* dst = reinterpret_cast<float*>(smem) + c * kBM + (warp & 3) * 32 + lane;
#pragma unroll
    for (int e = 0; e < 32; ++e) dst[e * kBM] = __uint_as_float(x[e]);
  }
  // Tensor memory is given back before the wait for the cluster's other CTAs: whoever waits for
  // some of it, a CTA that this one would wait for among them, waits for this CTA's own work alone.
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
  if (p.splits > 1) cg::this_cluster().sync();

  // ================================================================ epilogue: this CTA's rows
  // Eight columns a thread. (With two, 128 rows took 10000 cycles.)
  // The cluster's rank of the first CTA of this tile (the cluster is larger than the splits where one
  // launch computes both gradients).
  const uint32_t first_rank = cg::this_cluster().block_rank() - static_cast<uint32_t>(rank);
  const auto joined = [&](uint32_t at, float (&z)[8]) {  // lanes i .. i + 7 of a row, over all ranks
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p.splits == 1) {
        s = load_own(at + 16 * h);
      } else {
        for (int r0 = 0; r0 < p.splits; r0 += 4) {
          float4 v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (r0 + r < p.splits) v[r] = load_cluster(smem_at_rank(at + 16 * h, first_rank + r0 + r));
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (r0 + r < p.splits) s = make_float4(s.x + v[r].x, s.y + v[r].y, s.z + v[r].z, s.w + v[r].w);
        }
      }
      z[4 * h] = s.x;
      z[4 * h + 1] = s.y;
      z[4 * h + 2] = s.z;
      z[4 * h + 3] = s.w;
    }
  };
  if (col < p.cols) {  // (a multiple of 8)
    const bool wide = p.wide;
    float bias[8] = {};
    if (kForm == kCols && p.bias) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        bias[k] = p.bias_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.bias)[col + k])
                              : static_cast<const float*>(p.bias)[col + k];
    }
#pragma unroll 1
    for (int c = first; c < c1; c += kRowsOnce) {
      const int64_t row = static_cast<int64_t>(n0) + c;
      float add[8];
      if (kForm == kCols || kForm == kTurned) {
        unpack8(ahead[0], add);
#pragma unroll
        for (int k = 0; k + 1 < kAhead; ++k) ahead[k] = ahead[k + 1];
        ahead[kAhead - 1] = residual_of(c + kAhead * kRowsOnce);
      }
      float z[8];
      joined(sums + (c * kBM + i) * 4, z);
      if (kForm == kGated) {
        float u[8];
        joined(sums + (c * kBM + 64 + i) * 4, u);
        if (p.out[1]) {
          store8(p.out[1] + row * p.s_out[1] + col, true, z);
          store8(p.out[2] + row * p.s_out[2] + col, true, u);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] = activate(p.act, z[k]) * u[k];
      } else if (kForm == kCols) {
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] += bias[k];
        if (p.pre) store8(p.pre + row * p.s_pre + col, wide, z);
        if (p.act != DLM_ACT_NONE) {
#pragma unroll
          for (int k = 0; k < 8; ++k) z[k] = activate(p.act, z[k]);
        }
      }
      if (kForm == kCols || kForm == kTurned) {
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] += add[k];
      }
      const int o = kForm == kOuter ? second : 0;
      store8(p.out[o] + row * p.s_out[o] + col, wide, z);
    }
  }
  __syncwarp();
  if (p.splits > 1) cg::this_cluster().sync();  // nobody's sums go while others read them
}

// dW = dz^T x, 128 x 128 a tile, by `workers` CTAs. Not transposed: A is dz's columns, B those of x
// (both MN-major), and the sums go from tensor memory to the result, a row of it a lane, under the next
// tile's loads and MMAs (two accumulators). Stores of 32 bytes, whole sectors: 64 x 2048 x 8192 takes
// 10.9 us (33 MB at 4.07 TB/s, the rate of plain writes: 8.2), with stores of 16 bytes 14.6.
constexpr int kEpiWarp0 = 4;  // warps 4-7
__device__ __forceinline__ void few_weights(const Maps& maps, const Params& p, int worker, int workers) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Bars bars;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  constexpr int kStageBytes = 2 * kABytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&bars.full[s], 1);
      mbar_init(&bars.empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.acc_full[i], 1);
      mbar_init(&bars.acc_empty[i], 4);
    }
    mbar_init(&bars.done, 1);
    bars.abort = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    tmem_alloc(&bars.tmem_base, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem_base;
  volatile int* abort = &bars.abort;
  wait_for_previous();
  struct Tile {
    int second, row, col;
  };
  const auto tile_of = [&](int t) {
    const int strip = t % p.col_tiles, second = strip >= p.first_tiles;
    return Tile{second, (strip - second * p.first_tiles) * kBM, t / p.col_tiles * kBM};
  };
  if (warp == 0) {
    Ring ring;
    int fill = 0;
    bool ok = true, ready = true;
    for (int t = worker; ok && t < p.tiles; t += workers) {
      const Tile tl = tile_of(t);
      for (int kb = 0; kb < p.kblocks; ++kb, ++fill) {
        const int st = ring.stage;
        if (!warp_wait_if(ready, &bars.empty[st], ring.round ^ 1, abort, p.err, p.wait_ns)) {
          ok = false;
          break;
        }
        ring.next(p.stages);
        ready = fill + 1 < p.stages || mbar_test(&bars.empty[ring.stage], ring.round ^ 1);
        if (lane == 0) {
          uint8_t *a = smem + st * kStageBytes, *b = a + kABytes;
          uint64_t* bar = &bars.full[st];
          mbar_arrive_expect_tx(bar, kStageBytes);
          for (int i = 0; i < 2; ++i) tma_load_2d(a + i * kBoxBytes, &maps.b[tl.second], bar, tl.row + 64 * i, kb * kBK);
          for (int i = 0; i < 2; ++i) tma_load_2d(b + i * kBoxBytes, &maps.a[0], bar, tl.col + 64 * i, kb * kBK);
        }
      }
    }
    launch_dependents();
    if (lane == 0)  // every copy issued lands, whoever has given up
      for (int s = 0; s < p.stages; ++s) {
        const int n_s = fill > s ? (fill - s + p.stages - 1) / p.stages : 0;
        if (n_s) mbar_drain(&bars.full[s], (n_s - 1) & 1);
      }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t idesc = idesc_bf16_f32(kBM, kBM, true, true);
    const uint64_t a_desc0 = sdesc_sw128(smem_u32(smem), kBoxBytes, 1024), b_desc0 = sdesc_sw128(smem_u32(smem + kABytes), kBoxBytes, 1024);
    Ring ring;
    int tile = 0;
    bool ok = true, ready = false;
    for (int t = worker; ok && t < p.tiles; t += workers, ++tile) {
      const int acc = tile & 1;
      if (tile >= 2 && !warp_wait(&bars.acc_empty[acc], ((tile >> 1) - 1) & 1, abort, p.err, p.wait_ns)) break;
      tc_fence_after();
      for (int kb = 0; kb < p.kblocks; ++kb) {
        const int st = ring.stage;
        if (!warp_wait_if(ready, &bars.full[st], ring.round, abort, p.err, p.wait_ns)) {
          ok = false;
          break;
        }
        ring.next(p.stages);
        ready = mbar_test(&bars.full[ring.stage], ring.round);
        tc_fence_after();
        const uint32_t at = static_cast<uint32_t>(st) * (kStageBytes >> 4);
#pragma unroll
        for (int kk = 0; kk < kBK / 16; ++kk)
          mma_ss_elect(tmem + acc * kBM, a_desc0 + at + kk * 128, b_desc0 + at + kk * 128, idesc, (kb > 0 || kk > 0) ? 1u : 0u);
        mma_commit_elect(&bars.empty[st]);
      }
      if (!ok) break;
      mma_commit_elect(&bars.acc_full[acc]);
    }
    mma_commit_elect(&bars.done);
    mbar_drain(&bars.done, 0);
    __syncwarp();
  } else if (warp >= kEpiWarp0) {
    const int qw = warp & 3;
    int tile = 0;
    for (int t = worker; t < p.tiles; t += workers, ++tile) {
      const Tile tl = tile_of(t);
      const int acc = tile & 1;
      if (!warp_wait(&bars.acc_full[acc], (tile >> 1) & 1, abort, p.err, p.wait_ns)) break;
      tc_fence_after();
      const int64_t row = tl.row + qw * 32 + lane;
#pragma unroll 1
      for (int c = 0; c < kBM; c += 32) {
        uint32_t x[32];
        tmem_ld32(tmem + (static_cast<uint32_t>(qw * 32) << 16) + acc * kBM + c, x);
        tmem_wait_ld(x);
        if (c + 32 == kBM) {  // every column has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars.acc_empty[acc]);
        }
        const int n = min(32, p.cols - tl.col - c);  // (a multiple of 8)
        if (row < p.rows && n > 0) {
          __nv_bfloat16* dst = p.out[tl.second] + row * p.s_out[tl.second] + tl.col + c;
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) w[k] = pack_bf16x2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]));
          const auto sector = [&](__nv_bfloat16* to, int k) {  // 16 columns from the (2 k)th on
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[k]), "r"(w[k + 1]), "r"(w[k + 2]),
                         "r"(w[k + 3]), "r"(w[k + 4]), "r"(w[k + 5]), "r"(w[k + 6]), "r"(w[k + 7])
                         : "memory");
          };
          if (n == 32 && reinterpret_cast<uintptr_t>(dst) % 32 == 0) {
            sector(dst, 0);
            sector(dst + 16, 8);
          } else if (n == 32) {  // 16 bytes behind a sector's start
            *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
            sector(dst + 8, 4);
            *reinterpret_cast<uint4*>(dst + 24) = make_uint4(w[12], w[13], w[14], w[15]);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (8 * k < n) *reinterpret_cast<uint4*>(dst + 8 * k) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
          }
        }
        __syncwarp();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
}

__global__ void __launch_bounds__(kThreads, 2) few_weights_kernel(const __grid_constant__ Maps maps, const Params p) {
  few_weights(maps, p, static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
}

template <int kForm>
__global__ void __launch_bounds__(kThreads, 3) few_kernel(const __grid_constant__ Maps maps, const Params p) {
  few_product<kForm>(maps, p, static_cast<int>(blockIdx.x));
}

// Both gradients of a projection from dz: the first CTAs compute d x, those behind them dW. One
// reads the weights, the other writes as much: at the same time they use HBM both ways. 64 rows, 2048
// x 8192 with a gate: 35.5 us (134 MB, 3.8 TB/s with the element-wise part's launch), 43.2 in two launches.
__global__ void __launch_bounds__(kThreads, 2)
    few_gradients_kernel(const __grid_constant__ Maps x_maps, const Params x, const __grid_constant__ Maps w_maps, const Params w, int x_ctas,
                         int w_ctas) {
  const int block = static_cast<int>(blockIdx.x);
  if (block < x_ctas)
    few_product<kTurned>(x_maps, x, block);
  else if (block - x_ctas >= w_ctas)
    return;  // whole clusters are launched
  else if (w.splits > 1)
    few_product<kOuter>(w_maps, w, block - x_ctas);
  else
    few_weights(w_maps, w, block - x_ctas, w_ctas);
}

// ---------------------------------------------------------------- host side

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool aligned(const void* p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0; }

// What the plan leaves to fill in; the CTAs and their shared memory.
struct Launch {
  int64_t ctas;
  size_t smem;
};
Launch complete(Params* to, int64_t row_tiles, const FewPlan& plan, int room, int most = kMaxStages) {
  Params& p = *to;
  p.splits = plan.splits;
  // No more stages than steps, but room for the sums: where K is short, three CTAs fit on an SM.
  const int stage = kABytes + p.n * 128, steps = static_cast<int>(ceil_div(p.kblocks, p.splits));
  p.stages = room / stage < most ? room / stage : most;
  if (p.stages > steps) p.stages = steps;
  p.tmem_cols = p.n <= 32 ? 32 : p.n <= 64 ? 64 : 128;
  p.err = device_error_word();
  p.wait_ns = wait_budget_ns();
  const int sums = static_cast<int>(ceil_div(p.n, 32) * 32) * kBM * 4;
  return {row_tiles * p.col_tiles * p.splits, static_cast<size_t>(p.stages * stage > sums ? p.stages * stage : sums) + 1024};
}

// few_weights: as many CTAs as have tiles, up to `most`.
Launch complete_weights(Params* to, int room, int most) {
  Params& p = *to;
  p.splits = 1;
  p.tiles = static_cast<int>(ceil_div(p.cols, kBM)) * p.col_tiles;
  p.stages = room / (2 * kABytes);
  p.err = device_error_word();
  p.wait_ns = wait_budget_ns();
  return {p.tiles < most ? p.tiles : most, static_cast<size_t>(p.stages) * 2 * kABytes + 1024};
}

template <int kForm>
int launch_few(const Maps& m, Params p, int64_t row_tiles, const FewPlan& plan, cudaStream_t stream) {
  const auto kernel = few_kernel<kForm>;
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(kernel), kAloneRoom + 1024);
  Launch l = complete(&p, row_tiles, plan, kStageRoom);
  if (e == cudaSuccess && ceil_div(p.kblocks, p.splits) > p.stages) {
    // A deeper ring where an SM for each CTA is to be had, clusters and all.
    Params alone = p;
    const Launch la = complete(&alone, row_tiles, plan, kAloneRoom);
    if (la.ctas <= static_cast<int64_t>(p.splits) * active_clusters(reinterpret_cast<const void*>(kernel), p.splits, kThreads, kAloneRoom + 1024)) {
      p = alone;
      l = la;
    }
  }
  if (e == cudaSuccess)
    e = launch_overlapped(kernel, dim3(static_cast<unsigned>(l.ctas)), kThreads, l.smem, stream, p.splits, true, m, p);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "product launch: %s", cudaGetErrorString(e));
}

int operand_map(CUtensorMap* map, const Matrix& x, int box_rows) {
  return make_matrix_map(map, x.data, true, x.rows, x.cols, x.stride, box_rows);
}

}  // namespace

int64_t few_outer_ctas(int64_t rows, int64_t row_tiles, int matrices, const FewPlan& plan) {
  const int64_t tiles = row_tiles * matrices * ceil_div(rows, plan.splits > 1 ? plan.n : kBM);
  return plan.splits > 1 ? tiles * plan.splits : tiles < kSms ? tiles : kSms;
}

// Fitted to measured times (us): a launch, then for every round of two CTAs an SM the K steps
// (more each where two CTAs share an SM) and the rows of the epilogue, which cost more where other
// CTAs' sums are read (some 20 bytes a ns an SM from their shared memory); later rounds start with
// what the first one has done under the launch before. With splits one round only.
FewPlan plan_few(int64_t rows, int64_t row_tiles, int64_t kblocks, int matrices, bool outer, int splits, bool or_one) {
  constexpr double kStep[4] = {0.22, 0.225, 0.27, 0.35}, kShared[4] = {0.34, 0.36, 0.40, 0.50};  // n = 16, 32, 64, 128
  // Operands that L2 does not hold reach the SMs at some 12 TB/s in all, 32 KB a tile and K step of 128 x 128
  // (7471 x 520 x 6832: dx 164 us, dW 186; planned without it as 112 and 84).
  const double operands = static_cast<double>((outer ? matrices : 1) * rows + row_tiles * kBM) * static_cast<double>(kblocks) * kBK * 2;
  const auto least = [&](int64_t tiles, int n) {
    return operands < 80e6 ? 0.0 : 3.0 + static_cast<double>(tiles * kblocks) * (kABytes + n * kBK * 2) / 12e6;
  };
  FewPlan best = {128, 1, 1e300};
  for (int i = outer ? 2 : 0; i < 4; ++i) {
    const int n = 16 << i;
    if (n > 16 && n / 2 >= rows && !outer) break;
    for (int s = 1; s <= 8 && s <= kblocks; s *= 2) {
      if (splits && s != splits && !(or_one && s == 1)) continue;
      if (outer && s == 1) {  // few_weights
        if (n < 128) continue;
        const int64_t all = row_tiles * matrices * ceil_div(rows, n);
        const double tiles = static_cast<double>(all), k = static_cast<double>(kblocks), round = 0.5 * k > 0.92 ? 0.5 * k : 0.92;
        double us = 3.6 + 0.35 * k;                                        // an SM for each tile, six stages
        if (all > kSms) us = 3.0 + (tiles > 304 ? tiles / 304 : 1) * (k > 2 ? 1.3 + 0.38 * k : 2.2);  // two CTAs an SM, three stages
        if (splits) us = 3.5 + static_cast<double>(ceil_div(all, kSms)) * round;  // one an SM beside those of dx
        if (us < least(all, n)) us = least(all, n);
        if (us < best.us - 1e-9) best = {n, s, us};
        continue;
      }
      const int64_t ctas = row_tiles * matrices * ceil_div(rows, n) * s;
      if (s > 1 && ctas > (s > 2 ? kClustered : 2 * kSms)) break;
      const bool shared = ctas > kSms;
      const double rounds = static_cast<double>(ceil_div(ctas, 2 * kSms)), steps = static_cast<double>(ceil_div(kblocks, s));
      const double join = 0.5 + 0.06 * s + (n == 128 && s == 8 ? 3.0 : 0.0), epilogue = s == 1 ? 0.012 * n : join + 0.03 * n * (shared ? 2 : 1);
      double us = 3.0 + rounds * (steps * (shared ? kShared : kStep)[i] + epilogue) + 1.8 * (rounds - 1);
      if (us < least(ctas / s, n)) us = least(ctas / s, n);
      if (us < best.us - 1e-9) best = {n, s, us};
    }
  }
  return best;
}

int launch_few_gated(const GatedArgs& a, const FewPlan& plan, cudaStream_t stream) {
  Params p = {};
  p.rows = static_cast<int>(a.x.rows);
  p.cols = static_cast<int>(a.w_gate.rows);
  p.n = plan.n;
  p.col_tiles = p.first_tiles = static_cast<int>(ceil_div(p.rows, p.n));
  p.kblocks = p.first_kblocks = static_cast<int>(ceil_div(a.x.cols, kBK));
  p.act = a.act;
  p.wide = 1;
  const Matrix* outs[3] = {&a.out, &a.gate, &a.up};
  for (int i = 0; i < 3; ++i) {
    p.out[i] = static_cast<__nv_bfloat16*>(outs[i]->data);
    p.s_out[i] = outs[i]->stride;
  }
  Maps m = {};
  int st;
  if ((st = operand_map(&m.a[0], a.w_gate, 64)) != DLM_OK) return st;
  if ((st = operand_map(&m.a[1], a.w_up, 64)) != DLM_OK) return st;
  if ((st = operand_map(&m.b[0], a.x, p.n)) != DLM_OK) return st;
  return launch_few<kGated>(m, p, ceil_div(p.cols, 64), plan, stream);
}

namespace {

int set_up_cols(const Matrix* x, const Matrix* w, int runs, bool turned, const Epilogue& ep, const FewPlan& plan, Maps* maps, Params* to) {
  Params& p = *to;
  p.rows = static_cast<int>(x[0].rows);
  p.cols = static_cast<int>(turned ? w[0].cols : w[0].rows);
  p.n = plan.n;
  p.col_tiles = p.first_tiles = static_cast<int>(ceil_div(p.rows, p.n));
  p.first_kblocks = static_cast<int>(ceil_div(x[0].cols, kBK));
  p.kblocks = runs * p.first_kblocks;
  p.act = ep.act;
  p.bias = ep.bias;
  p.bias_bf16 = ep.bias_bf16;
  p.residual = static_cast<const __nv_bfloat16*>(ep.residual);
  p.out[0] = static_cast<__nv_bfloat16*>(ep.out);
  p.pre = static_cast<__nv_bfloat16*>(ep.pre);
  p.s_residual = ep.s_residual;
  p.s_out[0] = ep.s_out;
  p.s_pre = ep.s_pre;
  p.wide = aligned(p.out[0], p.s_out[0]) && (!p.residual || aligned(p.residual, p.s_residual)) && (!p.pre || aligned(p.pre, p.s_pre));
  int st;
  for (int i = 0; i < runs; ++i) {
    if ((st = operand_map(&maps->a[i], w[i], turned ? 64 : kBM)) != DLM_OK) return st;
    if ((st = operand_map(&maps->b[i], x[i], p.n)) != DLM_OK) return st;
  }
  return DLM_OK;
}

int set_up_outer(const Matrix* z, const Matrix& x, const Matrix* out, int count, const FewPlan& plan, Maps* maps, Params* to) {
  Params& p = *to;
  p.rows = static_cast<int>(z[0].cols);
  p.cols = static_cast<int>(x.cols);
  p.n = plan.splits > 1 ? plan.n : kBM;
  p.first_tiles = static_cast<int>(ceil_div(p.rows, p.n));
  p.col_tiles = count * p.first_tiles;
  p.kblocks = p.first_kblocks = static_cast<int>(ceil_div(x.rows, kBK));
  p.wide = 1;
  int st;
  for (int i = 0; i < count; ++i) {
    p.out[i] = static_cast<__nv_bfloat16*>(out[i].data);
    p.s_out[i] = out[i].stride;
    if ((st = operand_map(&maps->b[i], z[i], 64)) != DLM_OK) return st;
  }
  return operand_map(&maps->a[0], x, 64);
}

}  // namespace

int launch_few_cols(const Matrix* x, const Matrix* w, int runs, bool turned, const Epilogue& ep, const FewPlan& plan,
                    cudaStream_t stream) {
  Maps m = {};
  Params p = {};
  const int st = set_up_cols(x, w, runs, turned, ep, plan, &m, &p);
  if (st != DLM_OK) return st;
  const int64_t row_tiles = ceil_div(p.cols, kBM);
  return turned ? launch_few<kTurned>(m, p, row_tiles, plan, stream) : launch_few<kCols>(m, p, row_tiles, plan, stream);
}

int launch_few_outer(const Matrix* z, const Matrix& x, const Matrix* out, int count, const FewPlan& plan, cudaStream_t stream) {
  Maps m = {};
  Params p = {};
  const int st = set_up_outer(z, x, out, count, plan, &m, &p);
  if (st != DLM_OK) return st;
  if (plan.splits > 1) return launch_few<kOuter>(m, p, ceil_div(p.cols, kBM), plan, stream);
  // Six stages where a CTA has an SM to itself, three where two share one.
  const bool alone = ceil_div(p.cols, kBM) * p.col_tiles <= kSms;
  const Launch l = complete_weights(&p, alone ? kAloneRoom : kStageRoom, 2 * kSms);
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(few_weights_kernel), kAloneRoom + 1024);
  if (e == cudaSuccess)
    e = launch_overlapped(few_weights_kernel, dim3(static_cast<unsigned>(l.ctas)), kThreads, l.smem, stream, 1, true, m, p);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "product launch: %s", cudaGetErrorString(e));
}

int launch_few_gradients(const Matrix* z, const Matrix* w, int count, const Epilogue& ep, const FewPlan& x_plan, const Matrix& x,
                         const Matrix* dw, const FewPlan& w_plan, cudaStream_t stream) {
  Maps xm = {}, wm = {};
  Params xp = {}, wp = {};
  int st;
  if ((st = set_up_cols(z, w, count, true, ep, x_plan, &xm, &xp)) != DLM_OK) return st;
  if ((st = set_up_outer(z, x, dw, count, w_plan, &wm, &wp)) != DLM_OK) return st;
  const int64_t x_tiles = ceil_div(xp.cols, kBM), w_tiles = ceil_div(wp.cols, kBM);
  // (Four stages: with six of 16 rows what is read crowds out what is written: 40.2 us, not 37.7.)
  const Launch xl = complete(&xp, x_tiles, x_plan, kStageRoom, 4);
  const Launch wl = w_plan.splits > 1 ? complete(&wp, w_tiles, w_plan, kStageRoom) : complete_weights(&wp, kStageRoom, kSms);
  cudaError_t e = allow_smem(reinterpret_cast<const void*>(few_gradients_kernel), kStageRoom + 1024);
  const int64_t s = xp.splits, ctas = xl.ctas + ceil_div(wl.ctas, s) * s;
  if (e == cudaSuccess)
    e = launch_overlapped(few_gradients_kernel, dim3(static_cast<unsigned>(ctas)), kThreads, xl.smem > wl.smem ? xl.smem : wl.smem, stream,
                          xp.splits, true, xm, xp, wm, wp, static_cast<int>(xl.ctas), static_cast<int>(wl.ctas));
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "gradients launch: %s", cudaGetErrorString(e));
}

}  // namespace dlm
