// Head product for the log-probabilities of many rows (sx_head_logprobs with more rows than the weight-streaming kernel of
// sx_gemm_tc.cu takes): logits[r][n] = sum_k X[r][k] W[n][k], a dense contraction, and per row what the softmax needs of them.
//
// Two CTAs on neighbouring SMs share one product: 256 token rows (128 in each CTA, one per TMEM lane) by 256 vocabulary rows, of
// which each CTA holds half as the B operand - tcgen05.mma.cta_group::2, issued by the first CTA - so that an SM loads 32 KB
// for every 64 elements of K, two thirds of what a CTA of its own would need for the same tile.
//
// The tensor core's fp32 accumulator cuts off where a CPU rounds: every step of 16 elements of K loses up to an ulp of the
// running sum, always towards zero (measured: 6e-6 of a logit at K = 4096).  So no chain is longer than SX_SCORE_CHUNK_PAIR k-blocks: the
// epilogue adds the chunks' sums in registers, rounding to nearest, two TMEM accumulators in turn.  A thread of the epilogue owns a
// token row and half of the tile's columns; softmax sums and maxima of groups of 32 need no exchange between threads.
//
// Measured, 1000 rows, H = 4096, 151936 tokens (1.24 TFLOP): 0.92 ms by itself (1.35 PFLOP/s, 0.96 of what the library's product holds
// under the power cap, tensor pipe active 77-79 % of the cycles), 0.97-1.24 ms a call with the finishing kernel on different
// boxes.  Chains of 256 products instead of 512 cost 7 % more, of 384 2 % more, of 1024 6 % less.  Asking the L2 for weights 16 k-blocks ahead cost
// 3-14 %.
//
// Per CTA 320 threads: warp 0 TMA producer, warp 1 MMA issuer (the first CTA's; both hold the TMEM allocation), warps 2-9 epilogue.
// All waits are bounded as in sx_gemm_tc.cu; the CTAs of a pair leave together (cluster barriers before and after TMEM is freed).
#include <cuda.h>

#include <atomic>

#include "sx_kernels.cuh"
#include "sx_launch.cuh"
#include "sx_score.cuh"
#include "sx_tc_ptx.cuh"

#define PAIR_THREADS 320
#define PAIR_BK 64
#define PAIR_HALF (128 * PAIR_BK * 2)          // bytes of an operand half: 128 rows x 64 columns
#define PAIR_STAGE (2 * PAIR_HALF)
#define PAIR_STAGES 7
#define PAIR_SMEM (1024 + PAIR_STAGES * PAIR_STAGE + 256)

struct SxPairArgs {
  int R, V, num_kb, row_tiles, items, tiles;   // items: pairs of tiles (row tile fastest); tiles: of 128 vocabulary rows
  int w_tiled;
  uint32_t wait_limit;
  SxScoreOut sc;
  int32_t *status;
};

__device__ __forceinline__ uint32_t pair_addr(uint32_t local, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
  return a;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// Arrivals on the other CTA's barriers.  What they order is TMEM (by the tcgen05 fences) and what the TMA counts itself, so they
// need no release over the cluster: that waits for every store on its way, and tripled the time of the whole kernel.
__device__ __forceinline__ void pair_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// a box of one of the CTA's operand halves; its bytes count on the first CTA's barrier
__device__ __forceinline__ void pair_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2.L2::cache_hint"
      " [%0], [%1, {%3, %4}], [%2], %5;"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// arrives at the barrier of the same place in both CTAs once the MMAs issued so far are done
__device__ __forceinline__ void pair_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3) : "memory");
}

__global__ void __launch_bounds__(PAIR_THREADS, 1)
sx_score_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const SxPairArgs p) {
  extern __shared__ uint8_t pair_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)pair_raw + 1023) & ~(uintptr_t)1023);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + PAIR_STAGES * PAIR_STAGE);
  uint64_t *full = bars, *empty = bars + PAIR_STAGES, *tfull = bars + 2 * PAIR_STAGES, *tempty = tfull + 2;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(tempty + 2);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = blockIdx.x & 1;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  sx_pdl_launch_dependents();
  if (threadIdx.x == 0) {
    for (int i = 0; i < PAIR_STAGES; ++i) {
      mbar_init(smem_u32(&full[i]), 2);             // the producers of both CTAs, and their bytes
      mbar_init(smem_u32(&empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&tfull[i]), 1);
      mbar_init(smem_u32(&tempty[i]), 16);          // the epilogue warps of both CTAs
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  pair_sync();                                      // both CTAs' barriers exist
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      // As in sx_gemm_tc.cu: the weights of the first stages are requested before the wait on the preceding kernel (pass 0), the
      // rows of those stages behind it (pass 1), then both together (pass 2).
      // (The weights are not marked evict-first as they are there: the row tiles read them at about the same time, one of
      // them from memory.)
      uint64_t pol_w;
      asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol_w));
      const uint64_t pol_x = policy_evict_last();
      bool ok = true;
      for (int pass = 0; pass < 3 && ok; ++pass) {
        if (pass == 1) sx_pdl_wait();
        int stage = 0, cnt = 0;
        uint32_t phase = 0;
        for (int item = pair; item < p.items && ok; item += pairs) {
          const int vt = item / p.row_tiles, rt = item - vt * p.row_tiles;
          const int wt = vt * 2 + (int)rank, row = rt * 256 + (int)rank * 128;
          for (int kb = 0; kb < p.num_kb; ++kb, ++cnt) {
            if (pass < 2 && cnt >= PAIR_STAGES) break;
            const uint32_t fb = pair_addr(smem_u32(&full[stage]), 0);
            const uint32_t a = smem_u32(smem + (size_t)stage * PAIR_STAGE), b = a + PAIR_HALF;
            const bool want = pass == 2 ? cnt >= PAIR_STAGES : true;
            if (pass == 2 && want && !mbar_wait(smem_u32(&empty[stage]), phase ^ 1u, abort_flag, p.wait_limit)) { ok = false; break; }
            if (want && pass != 1) {
              pair_expect(fb, PAIR_STAGE);
              pair_load(b, &tmW, fb, p.w_tiled ? 0 : kb * PAIR_BK, p.w_tiled ? (wt * p.num_kb + kb) * 128 : wt * 128, pol_w);
            }
            if (want && pass != 0) pair_load(a, &tmX, fb, kb * PAIR_BK, row, pol_x);
            if (++stage == PAIR_STAGES) { stage = 0; phase ^= 1u; }
          }
          if (pass < 2 && cnt >= PAIR_STAGES) break;
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // fp32 accumulate, bf16 A and B, both K-major, N = 256, M = 256 over the pair
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int item = pair; item < p.items && ok; item += pairs) {
        for (int kb0 = 0; kb0 < p.num_kb && ok; kb0 += SX_SCORE_CHUNK_PAIR) {
          const int kb1 = min(p.num_kb, kb0 + SX_SCORE_CHUNK_PAIR);
          if (!mbar_wait(smem_u32(&tempty[acc]), acc_phase ^ 1u, abort_flag, p.wait_limit)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + (uint32_t)(acc * 256);
          for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait(smem_u32(&full[stage]), phase, abort_flag, p.wait_limit)) { ok = false; break; }
            tc_fence_after();
            const uint32_t a = smem_u32(smem + (size_t)stage * PAIR_STAGE), b = a + PAIR_HALF;
#pragma unroll
            for (int k = 0; k < PAIR_BK / 16; ++k)
              pair_mma(d_tmem, smem_desc(a + k * 32), smem_desc(b + k * 32), idesc, (kb > kb0 || k > 0) ? 1u : 0u);
            pair_commit(smem_u32(&empty[stage]));
            if (++stage == PAIR_STAGES) { stage = 0; phase ^= 1u; }
          }
          if (!ok) break;
          pair_commit(smem_u32(&tfull[acc]));
          if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;   // TMEM lane quarter, half of the columns
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    sx_pdl_wait();
    for (int item = pair; item < p.items && ok; item += pairs) {
      const int vt = item / p.row_tiles, rt = item - vt * p.row_tiles;
      const int row = rt * 256 + (int)rank * 128 + q * 32 + lane;
      float v[128];
#pragma unroll
      for (int j = 0; j < 128; ++j) v[j] = 0.f;
      for (int kb0 = 0; kb0 < p.num_kb; kb0 += SX_SCORE_CHUNK_PAIR) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&tfull[acc]), acc_phase, abort_flag, p.wait_limit));
        if (!ok) break;
        tc_fence_after();
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * 256 + half * 128);
#pragma unroll
        for (int c = 0; c < 128; c += 16) {
          float x[16];
          tc_ld16(taddr + c, x);
#pragma unroll
          for (int j = 0; j < 16; ++j) v[c + j] += x[j];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) pair_arrive(pair_addr(smem_u32(&tempty[acc]), 0));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok) break;
      const int n0 = vt * 256 + half * 128;                     // first vocabulary row of this thread's columns
      if (n0 + 128 > p.V) {
#pragma unroll
        for (int j = 0; j < 128; ++j)
          if (n0 + j >= p.V) v[j] = -INFINITY;
      }
      const int tile = vt * 2 + half;
      float gm[4], mx = -INFINITY;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        gm[g] = v[g * 32];
#pragma unroll
        for (int j = 1; j < 32; ++j) gm[g] = fmaxf(gm[g], v[g * 32 + j]);
        mx = fmaxf(mx, gm[g]);
      }
      if (tile < p.tiles && row < p.R) {
#pragma unroll
        for (int j = 0; j < 128; j += 8) sx_store8<true>(p.sc.logits + sx_score_at(p.sc, row, n0 + j), v + j);
        *reinterpret_cast<float4 *>(p.sc.maxima + ((size_t)tile * p.sc.rows + row) * 4) = make_float4(gm[0], gm[1], gm[2], gm[3]);
        const float ref = mx > -INFINITY ? mx : 0.f;
        float2 s2 = make_float2(0.f, 0.f), t2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 128; j += 2) score_pair(make_float2(v[j], v[j + 1]), p.sc.scale, ref, s2, t2);
        float *out = p.sc.sums + ((size_t)tile * p.sc.rows + row) * 3;
        out[0] = mx;
        out[1] = s2.x + s2.y;
        out[2] = t2.x + t2.y;
      }
      __syncwarp();
    }
  }
  // the common exit: copies in flight land, then both CTAs have stopped using each other's memory, then TMEM is freed
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0) sx_set_status(p.status, SX_ERR_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(20000);
  }
  tc_fence_before();
  __syncthreads();
  pair_sync();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
  __syncthreads();
  pair_sync();
}

// ---- host side -------------------------------------------------------------------------------------------------------------
// pairs of CTAs that the current device holds at a time
static sx_status pairs_of_device(int *pairs) {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return SX_ERR_CUDA;
  if (dev < 64 && (n = known[dev].load(std::memory_order_acquire)) > 0) { *pairs = n; return SX_OK; }
  if (cudaFuncSetAttribute(sx_score_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PAIR_SMEM) != cudaSuccess) return SX_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(2 * 1024);
  cfg.blockDim = dim3(PAIR_THREADS);
  cfg.dynamicSmemBytes = PAIR_SMEM;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 2;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, sx_score_pair_kernel, &cfg) != cudaSuccess || n < 1) return SX_ERR_CUDA;
  if (dev < 64) known[dev].store(n, std::memory_order_release);
  *pairs = n;
  return SX_OK;
}

sx_status sx_launch_score_pairs(const bf16 *W, bool tiled, int V, int K, const bf16 *X, int R, const SxScoreOut &out, int *parts,
                                int32_t *status, cudaStream_t st) {
  if (K % 8 != 0 || R < 1 || R > out.rows) return SX_ERR_UNSUPPORTED;
  int pairs = 0;
  SX_TRY(pairs_of_device(&pairs));
  SxPairArgs p;
  memset(&p, 0, sizeof(p));
  p.R = R; p.V = V; p.num_kb = (K + PAIR_BK - 1) / PAIR_BK;
  p.row_tiles = (R + 255) / 256;
  p.tiles = (V + SX_TILE_M - 1) / SX_TILE_M;
  p.items = (p.tiles + 1) / 2 * p.row_tiles;
  p.w_tiled = tiled ? 1 : 0;
  p.wait_limit = SX_WAIT_LIMIT;
  p.sc = out;
  p.status = status;
  CUtensorMap mw, mx;
  if (!sx_weight_map(W, V, K, tiled, &mw) || !sx_tma_map_2d(X, R, K, 128, &mx)) return SX_ERR_CUDA;
  *parts = p.tiles;
  if (pairs > p.items) pairs = p.items;
  return sx_rc(sx_launch_cluster(sx_score_pair_kernel, dim3(2 * pairs), dim3(PAIR_THREADS), PAIR_SMEM, 2, st, mw, mx, p));
}
