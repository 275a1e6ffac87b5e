// Decode attention over the 8-bit paged cache on the 5th-generation tensor cores, for head dimension 128 and many
// queries per KV head: a prefix that a group of sequences shares (its members' queries side by side), or the
// sibling rows of a draft tree.  Up to 128 queries per tile.
//
// Work, partial results and merge are those of sx_attn8.cuh: a CTA takes one run of 128-slot blocks.  Per block, with the
// queries on M:
//     S[q][slot] = sum_d Q[q][d] kc[slot][d]         A = Q, B = K codes as they lie in the pages (both K-major)
//     O[q][d]   += sum_slot P[q][slot] V[slot][d]    A = P from tensor memory, B = V as bf16 (N-major)
// First product: a bf16 query, its row scaled by a power of two, is the sum of an e4m3 and an e5m2 number (a8_split); so A is
// [high part] then [low part] into the same accumulator - the cost of one bf16 product, and K is used as it was stored;
// its scale is a factor of the slot's scores.  Second product: weights need 16 bits (in 8 a long flat tail of small weights
// would vanish), so V becomes bf16 in shared memory, exactly (4 significand bits, a power of two), by eight warps of
// their own, once per block whatever the number of queries: a code's exponent and mantissa are moved to their places in a
// bf16 number and one packed multiplication by 2^(120 + e - A8_V_SHIFT) puts bias and scale right.  The shift leaves room
// for the sums: weights reach 2^T8_SLACK and values 2^129, and without it 600 slots of 2^110 whose scores rise became
// infinity - infinity; with it 2^19 slots of any values are held, and the smallest codes of the smallest scale, 2^-117, are
// still normal numbers.
// (Tried before: slots on M, so that a thread owned a slot and the softmax ran across threads - a barrier vote per block,
// weights through shared memory, a reference per query to fetch for every score: 6500 cycles per block with 128 queries,
// 3400 with 32.  V as fp16 codes with its scale in the score and a second factor in the sums: three broadcasts from
// shared memory per score pair, 4000 cycles.  K as bf16 too: the widening of both took 4700.)
//
// Two groups of four softmax warps take a half of every block each (64 slots), with scores (two buffers: the next
// block's are ready when a group comes to them), weights (in place of the scores, as they are read), references, sums and
// an output accumulator of their own: 2 x (2 x 64 + 128) columns of tensor memory, and nothing to agree on between
// threads - a thread owns one query, its reference and its sum, and moves the reference when a score exceeds it by
// more than 2^T8_SLACK.  With up to 64 (32) queries the 128 rows of the products hold 2 (4) copies of them, and a
// copy's threads take a half (a quarter) of the group's slots, with weights of zero for the others: the products cost the
// same, and the softmax of 32 queries, one warp's work before, is spread over four.  At the end of a segment the groups'
// results, which lie in the same rows of tensor memory, become one; every copy leaves its own.
//
// Measured: 2700 to 3100 cycles per block with 128 queries (the softmax warps: two thirds of the issue slots, half of the
// exponential unit), 2450 with 32 (the chain first product, softmax, second product, beside the widening of V), 5 us to the
// first block and 3 to 5 us for the end of a segment.  4 x 32768 slots of 8 heads under 32 queries: 98 us with the merge in a
// graph of calls, 2.8 TB/s (108 us as a call of its own); a prefix of 30001 slots under 256 queries, own slots and merge: 96 us,
// 345 TFLOP/s.
//
// Warps: 0 K producer, 1 issuer of the first product (owns TMEM), 2 V producer, 3 issuer of the second, 4-11 softmax,
// 12-19 widen V, lay out the scales of K and load Q.  Every mbarrier wait is bounded (sx_tc_ptx.cuh).
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>

#include "sx_attn8.cuh"
#include "sx_kernels.cuh"
#include "sx_launch.cuh"
#include "sx_tc_ptx.cuh"

#define T8_THREADS 640
#define T8_BLK (128 * 128)               // bytes of the codes of a block
#define T8_NONE (-3e38f)                 // reference before the first visible score
// Weights are bf16, sums fp32: their precision does not depend on where the reference lies, so it moves only where the
// range of numbers asks for it: 2^T8_SLACK below, 2^129 for a value, 2^19 slots and A8_V_SHIFT off fill fp32 to the top, and
// what falls off its bottom is below 2^-105 (values of 1 behind a sink of zeros 72 nats above).
#define T8_SLACK 24.f
#define T8_NK 4                          // ring slots of 16 KB for the codes of K,
#define T8_NV 3                          // of V
#define T8_NW 2                          // bf16 copies (32 KB) of V blocks
#define T8_NC 4                          // entries of K scales; of query factors
#define T8_Q_BYTES T8_BLK                // one of the two parts
#define T8_O_COL 256                     // tensor memory: scores / weights of the groups, then their outputs
#define T8_OFF_W (2 * T8_Q_BYTES)
#define T8_OFF_RING (T8_OFF_W + T8_NW * 2 * T8_BLK)
#define T8_OFF_SC (T8_OFF_RING + (T8_NK + T8_NV) * T8_BLK)             // [slot of V][128 + 128] exponent bytes of K and V
#define T8_OFF_KS (T8_OFF_SC + 1024)                     // [entry][128] scales of K
#define T8_OFF_QF (T8_OFF_KS + T8_NC * 512)              // [entry][128] factor of the query's scores
#define T8_OFF_ML (T8_OFF_QF + T8_NC * 512)              // [group][128] (reference, sum) at the end of a segment
#define T8_OFF_BAR (T8_OFF_ML + 2048)
#define T8_OFF_PLAN (T8_OFF_BAR + 512)
#define T8_FIXED (T8_OFF_PLAN + 1024)                    // + alignment
#define T8_SMEM_MAX (227 * 1024)

template <int N> __device__ __forceinline__ void t8_setreg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void t8_setreg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ float t8_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
#define T8_WAIT_POLLS (1u << 17)          // x SX_NAP_NS: 2.6 s at most
// true in one thread of the warp; unlike a test of the lane, the compiler knows that of it, and issues the tensor-core
// instructions (whose operands live in uniform registers) without a loop over the threads that might be there
__device__ __forceinline__ bool t8_elect() {
  uint32_t one;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ float t8_max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// two fp32 operations in one instruction
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 t8_pack(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void t8_unpack(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 t8_mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 t8_add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 t8_fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// D[tmem] (+)= A[smem] * B[smem], 8-bit x 8-bit -> fp32, M = 128, K = 32
__device__ __forceinline__ void t8_mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], bf16 x bf16 -> fp32, M = 128, K = 16
__device__ __forceinline__ void t8_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// columns of this thread's TMEM lane as they are
__device__ __forceinline__ void t8_st(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void t8_st(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void t8_ld(uint32_t taddr, float (&v)[16]) { tc_ld16(taddr, v); }
__device__ __forceinline__ void t8_ld(uint32_t taddr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31 "
      "}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void t8_ld(uint32_t taddr, float (&v)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, "
      "%42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, "
      "%62, %63 "
      "}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
        "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]),
        "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
        "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]),
        "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
      : "r"(taddr) : "memory");
}
// four codes to bf16, times `f` (a packed pair of equal bf16 numbers): exponent and mantissa move to the low end of the
// exponent's place and the high end of the mantissa's, which is the value times 2^-120; f = 2^(120 + e - A8_V_SHIFT)
__device__ __forceinline__ void t8_widen4(uint32_t x, uint32_t f, uint32_t &lo2, uint32_t &hi2) {
  const uint32_t hi = ((x >> 4) & 0x07070707u) | (x & 0x80808080u), lo = (x << 4) & 0xf0f0f0f0u;
  uint32_t a = __byte_perm(lo, hi, 0x5140), b = __byte_perm(lo, hi, 0x7362);
  const __nv_bfloat162 ff = *reinterpret_cast<const __nv_bfloat162 *>(&f);
  __nv_bfloat162 va = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&a), ff), vb = __hmul2(*reinterpret_cast<__nv_bfloat162 *>(&b), ff);
  lo2 = *reinterpret_cast<uint32_t *>(&va);
  hi2 = *reinterpret_cast<uint32_t *>(&vb);
}
// packed bf16 2^n, n in [-126, 127]
__device__ __forceinline__ uint32_t t8_pow2x2(int n) { return (uint32_t)(127 + n) * 0x00800080u; }
__device__ __forceinline__ uint32_t t8_mulx2(uint32_t x, uint32_t f) {
  const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&f));
  return *reinterpret_cast<const uint32_t *>(&v);
}

// exponent bytes of rows of zeros, for boxes without slots or without a page (not what the ring held before)
#define T8_16(b) b, b, b, b, b, b, b, b, b, b, b, b, b, b, b, b
__device__ __align__(16) const uint8_t t8_zero_row_bytes[128] = {T8_16(127), T8_16(127), T8_16(127), T8_16(127),
                                                                 T8_16(127), T8_16(127), T8_16(127), T8_16(127)};

template <bool PRE, int COPIES>
__global__ void __launch_bounds__(T8_THREADS, 1)
sx_attn8_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                   const __grid_constant__ SxA8 p, int slab, uint32_t wait_limit) {
  constexpr int NK = T8_NK, NV = T8_NV, NW = T8_NW;
  extern __shared__ uint8_t t8_raw[];
  // an offset, not a cast to an integer and back: the compiler keeps seeing shared memory (generic loads cost a multiple)
  uint8_t *smem = t8_raw + ((0u - smem_u32(t8_raw)) & 1023u);
  uint8_t *sQ = smem, *sW = smem + T8_OFF_W, *ringK = smem + T8_OFF_RING, *ringV = ringK + NK * T8_BLK;
  uint8_t *sc = smem + T8_OFF_SC;
  float *ks_sh = reinterpret_cast<float *>(smem + T8_OFF_KS), *qf = reinterpret_cast<float *>(smem + T8_OFF_QF);
  float2 *ml_sh = reinterpret_cast<float2 *>(smem + T8_OFF_ML);
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + T8_OFF_BAR);
  uint64_t *kfull = bars, *kempty = kfull + NK, *vfull = kempty + NK, *vempty = vfull + NV;
  // [group][block & 1]: scores ready, weights ready, second product done
  uint64_t *sfull = vempty + NV, *pfull = sfull + 4, *pvdone = pfull + 4, *ofree = pvdone + 4, *wfull = ofree + 2;
  uint64_t *wempty = wfull + NW, *cfull = wempty + NW, *qfull = cfull + T8_NC, *qempty = qfull + 1, *xfull = qempty + 1;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(xfull + 1);
  static_assert(COPIES == 1 || COPIES == 2 || COPIES == 4, "rows of a product hold whole copies");
  constexpr int QT = 128 / COPIES, CH = 64 / COPIES;       // queries of a copy; its slots of a group's half
  // A product of codes reaches 2^25 and a scale of K 2^120, which fp32 does not hold.  With 128 queries part of the scale is
  // left to the query's factor; with fewer both factors are multiplied first, which needs no shift and is done before the
  // product arrives (tree 98 against 101 us; but a prefix under 256 queries 98 against 96 us).
  constexpr bool FACTORS_FIRST = COPIES > 1;
  constexpr float K_SHIFT = FACTORS_FIRST ? 1.f : 131072.f;
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  a8_enter<PRE>(p);
  const SxA8List &ls = PRE ? p.pre : p.own;
  A8Plan pl;
  a8_plan<PRE, T8_THREADS>(p, ls, slab, smem + T8_OFF_PLAN, pl);
  a8_planned<PRE>(p);
  a8_publish<PRE, T8_THREADS>(p, pl, ls);
  const int total = pl.cum[pl.units], g0 = (int)min((int64_t)total, (int64_t)blockIdx.x * pl.per), g1 = g0 + min(total - g0, pl.per);
  if (g0 >= g1) { a8_leave<PRE>(p); return; }
  const int nblk = g1 - g0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NK; ++i) { mbar_init(smem_u32(&kfull[i]), 1); mbar_init(smem_u32(&kempty[i]), 1); }
    for (int i = 0; i < NV; ++i) { mbar_init(smem_u32(&vfull[i]), 1); mbar_init(smem_u32(&vempty[i]), 4); }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&sfull[i]), 1); mbar_init(smem_u32(&pfull[i]), 4); mbar_init(smem_u32(&pvdone[i]), 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&ofree[i]), 8);
    for (int i = 0; i < NW; ++i) { mbar_init(smem_u32(&wfull[i]), 4); mbar_init(smem_u32(&wempty[i]), 1); }
    for (int i = 0; i < T8_NC; ++i) mbar_init(smem_u32(&cfull[i]), 4);
    mbar_init(smem_u32(qfull), 8);
    mbar_init(smem_u32(qempty), 1);
    mbar_init(smem_u32(xfull), 8);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tc_alloc(smem_u32(tmem_slot), 512);
    tc_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) {
    t8_setreg_dec<56>();
    if (warp == 0 || warp == 2) {
      // ---- producers: the codes of a block (one box per `slab` slots, which lie in one page); V's with the exponent bytes ----
      const bool is_v = warp == 2;
      const CUtensorMap *map = is_v ? &tmV : &tmK;
      uint8_t *ring = is_v ? ringV : ringK;
      uint64_t *full = is_v ? vfull : kfull, *empty = is_v ? vempty : kempty;
      const int depth = is_v ? NV : NK, nbox = 128 / slab;
      const uint64_t pol = policy_evict_first();
      bool bad = false;
      A8Seg s = a8_seek<PRE>(p, pl, ls, slab, g0);
      // first pool row of box `lane` of the block at list position x; -1 where there is none
      auto row_of = [&](int x) -> int {
        if (lane >= nbox) return -1;
        const int slot = s.first + (x - s.x0) * 128 + lane * slab;
        if (slot >= s.end) return -1;
        const int lp = slot / p.page, off = slot - lp * p.page;
        const int pp = lp < p.max_pages ? p.page_table[(int64_t)s.b0 * p.max_pages + lp] : -1;
        if (pp < 0 || pp >= p.num_pages) { bad = true; return -1; }
        return (pp * p.nkv + s.h) * p.page + off;
      };
      int row = row_of(g0);
#pragma unroll 1
      for (int li = 0; li < nblk; ++li) {
        int next = -1;
        if (li + 1 < nblk) {                                // looked up while this block's slot may still be busy
          if (g0 + li + 1 == s.x1) s = a8_seek<PRE>(p, pl, ls, slab, g0 + li + 1);
          next = row_of(g0 + li + 1);
        }
        const int slot = li % depth;
        if (li >= depth && !mbar_wait_warp(&empty[slot], (uint32_t)(li / depth - 1) & 1u, abort_flag, wait_limit, lane)) break;
        const uint32_t fb = smem_u32(&full[slot]);
        if (lane == 0) mbar_expect_tx(fb, T8_BLK + (is_v ? 256u : 0u));
        __syncwarp();
        if (lane < nbox) {
          // a box behind the last row of the pool reads zeros
          tma_load_2d(smem_u32(ring + slot * T8_BLK + lane * slab * 128), map, fb, 0, row >= 0 ? row : p.num_pages * p.nkv * p.page, pol);
          if (is_v) {
            bulk_load(smem_u32(sc + slot * 256 + lane * slab), row >= 0 ? p.ks + row : t8_zero_row_bytes, (uint32_t)slab, fb);
            bulk_load(smem_u32(sc + slot * 256 + 128 + lane * slab), row >= 0 ? p.vs + row : t8_zero_row_bytes, (uint32_t)slab, fb);
          }
        }
        row = next;
      }
      if (!is_v && __any_sync(0xffffffffu, bad) && lane == 0) sx_set_status(p.status, SX_ERR_CAPACITY);
    } else if (t8_elect()) {
      A8Seg s = a8_seek<PRE>(p, pl, ls, slab, g0);
      int item = 0, seg_li = 0;                             // segment number, its first block in the run
      const uint32_t acc32 = (1u << 4) | (8u << 24);        // fp32 accumulate, M = 128 (M / 16 at bit 24)
      if (warp == 1) {
        // ---- first product: e4m3 (format 0; the low parts of A e5m2, format 1 at bit 7), both operands K-major, N = 64 (N / 8 at
        // bit 17)
        const uint64_t qd = smem_desc(smem_u32(sQ));
        bool ok = true;
#pragma unroll 1
        for (int li = 0; li < nblk && ok; ++li) {
          if (li > 0 && g0 + li == s.x1) { s = a8_seek<PRE>(p, pl, ls, slab, g0 + li); ++item; seg_li = li; }
          if (li == seg_li && !mbar_wait_nap(qfull, (uint32_t)item & 1u, abort_flag, wait_limit)) break;
          const int slot = li % NK, b = li & 1;
          if (!mbar_wait_nap(&kfull[slot], (uint32_t)(li / NK) & 1u, abort_flag, wait_limit)) break;
          // the scales too: whoever sees the scores may read them
          if (!mbar_wait_nap(&cfull[li % T8_NC], (uint32_t)(li / T8_NC) & 1u, abort_flag, wait_limit)) break;
          const uint64_t kd = smem_desc(smem_u32(ringK + slot * T8_BLK));
#pragma unroll 1
          for (int g = 0; g < 2 && ok; ++g) {
            // the weights of the group's block before last, which lie in place of its scores, have met V
            if (li >= 2) ok = mbar_wait_nap(&pvdone[g * 2 + b], (uint32_t)((li >> 1) - 1) & 1u, abort_flag, wait_limit);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < 8; ++k)
              t8_mma_f8(tmem + (uint32_t)(g * 128 + b * 64), qd + (uint64_t)(((k >> 2) * T8_Q_BYTES + (k & 3) * 32) >> 4),
                        kd + (uint64_t)((g * (T8_BLK / 2) + (k & 3) * 32) >> 4), acc32 | (8u << 17) | (k < 4 ? 0u : 1u << 7), k > 0 ? 1u : 0u);
            tc_commit(smem_u32(&sfull[g * 2 + b]));
          }
          tc_commit(smem_u32(&kempty[slot]));
          if (g0 + li + 1 == s.x1) tc_commit(smem_u32(qempty));       // the segment's queries are not needed any more
        }
      } else {
        // ---- second product: bf16 (format 1), weights from tensor memory, V N-major, N = 128 --------------------------
        bool ok = true;
#pragma unroll 1
        for (int li = 0; li < nblk && ok; ++li) {
          if (li > 0 && g0 + li == s.x1) { s = a8_seek<PRE>(p, pl, ls, slab, g0 + li); ++item; seg_li = li; }
          const int wb = li % NW, b = li & 1;
          const bool first = li == seg_li;
          if (!mbar_wait_nap(&wfull[wb], (uint32_t)(li / NW) & 1u, abort_flag, wait_limit)) break;
          const uint64_t wd = smem_desc_mn(smem_u32(sW + wb * 2 * T8_BLK), T8_BLK, 1024u);
#pragma unroll 1
          for (int g = 0; g < 2 && ok; ++g) {
            ok = mbar_wait_nap(&pfull[g * 2 + b], (uint32_t)(li >> 1) & 1u, abort_flag, wait_limit);
            // the group has read out its output of the segment before
            if (ok && first && item > 0) ok = mbar_wait_nap(&ofree[g], (uint32_t)(item - 1) & 1u, abort_flag, wait_limit);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < 4; ++k)
              t8_mma_ta(tmem + T8_O_COL + (uint32_t)g * 128u, tmem + (uint32_t)(g * 128 + b * 64 + k * 8),
                        wd + (uint64_t)((g * 4 + k) * 128),
                        acc32 | (1u << 7) | (1u << 10) | (1u << 16) | (16u << 17), (first && k == 0) ? 0u : 1u);
            tc_commit(smem_u32(&pvdone[g * 2 + b]));
          }
          tc_commit(smem_u32(&wempty[wb]));
        }
      }
    }
  } else if (warp >= 12) {
    // ---- V codes to bf16 ([64 columns][128 slots][128 bytes] twice, 128-byte swizzle), scales of K, queries --------------
    t8_setreg_dec<80>();
    // Two teams of four warps take the blocks in turn, each with its copy of V; the queries of every segment are loaded by
    // both, half of the rows each (a team alone, row after row, kept a segment's first block waiting for 4 us)
    const int team = (warp - 12) >> 2, tid = threadIdx.x & 127, c = tid & 7, r0 = tid >> 3;
    A8Seg s = a8_seek<PRE>(p, pl, ls, slab, g0);
    int item = -1;
    bool ok = true;
#pragma unroll 1
    for (int li = team;; li += 2) {
      const int at_x = g0 + min(li, nblk - 1);
#pragma unroll 1
      while (ok && (item < 0 || at_x >= s.x1)) {
        // both teams wait for the end of every segment's first products, so that neither can be a phase behind
        if (item >= 0) {
          ok = mbar_wait_warp(qempty, (uint32_t)item & 1u, abort_flag, wait_limit, lane);
          s = a8_seek<PRE>(p, pl, ls, slab, s.x1);
        }
        ++item;
        // the two parts (rows of 128 bytes, 128-byte swizzle) and factor; eight threads share a row
        const int buf = item % T8_NC;
        {
          const int q0 = team * 64 + r0;
          uint4 xs[4][2];                                     // four rows on the way together
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int query = (q0 + k * 16) % QT;
            const bool live = query < s.cols;
            const int qi = s.tile * QT + (live ? query : 0), j = qi / p.G, r = s.r0 + j;
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (int64_t)r * p.q_stride + (int64_t)(s.h * p.G + qi - j * p.G) * 128 + c * 16);
            xs[k][0] = live ? src[0] : make_uint4(0, 0, 0, 0);
            xs[k][1] = live ? src[1] : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int row = 0; row < 4; ++row) {
            const int q = q0 + row * 16;
            const uint4 *x = xs[row];
            const uint32_t m = 0x7fff7fffu;
            uint32_t top = __vmaxu2(__vmaxu2(__vmaxu2(x[0].x & m, x[0].y & m), __vmaxu2(x[0].z & m, x[0].w & m)),
                                    __vmaxu2(__vmaxu2(x[1].x & m, x[1].y & m), __vmaxu2(x[1].z & m, x[1].w & m)));
            top = max(top & 0xffffu, top >> 16);
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o, 8));
            // largest magnitude into (224, 448], as for the rows of the cache
            const int e = (int)(top >> 7);
            int ex = top == 0 || e == 255 ? 0 : e - 135 + ((top & 0x7f) > 96 ? 1 : 0);
            ex = max(-126, ex);
            const float up = __uint_as_float((uint32_t)(127 - ex) << 23);
            const uint32_t in[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float2 f = make_float2(__uint_as_float(in[k] << 16) * up, __uint_as_float(in[k] & 0xffff0000u) * up);
              uint32_t h2, l2;
              a8_split(f, e != 255, h2, l2);
              if (k & 1) { hi[k >> 1] |= h2 << 16; lo[k >> 1] |= l2 << 16; }
              else { hi[k >> 1] = h2; lo[k >> 1] = l2; }
            }
            uint8_t *at = sQ + q * 128 + ((c ^ (q & 7)) << 4);
            *reinterpret_cast<uint4 *>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4 *>(at + T8_Q_BYTES) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            // (held to finite numbers: under a query that large every score is beyond telling apart)
            if (c == 0) {
              const float f = __uint_as_float((uint32_t)(127 + ex) << 23) * p.scale_log2 * K_SHIFT;
              qf[buf * 128 + q] = fminf(fmaxf(f, -FLT_MAX), FLT_MAX);
            }
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(qfull));
      }
      if (!ok || li >= nblk) break;
      const int slot = li % NV, e = li % T8_NC;
      if (!mbar_wait_warp(&vfull[slot], (uint32_t)(li / NV) & 1u, abort_flag, wait_limit, lane)) break;
      const uint8_t *kbytes = sc + slot * 256, *vbytes = kbytes + 128;
      // a row of K or V that is not finite makes the slot's scores so (whoever sees the slot gets it, whoever does not is
      // spared); such a V is zero here
      const int kbyte = kbytes[tid], vbyte = vbytes[tid];
      ks_sh[e * 128 + tid] = kbyte == 255 || vbyte == 255 ? __int_as_float(0x7fffffff) : a8_pow2(kbyte) * (1.f / K_SHIFT);
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&cfull[e]));
      // Chunks 2c and 2c + 1 of the half; the lanes of the second half go the other way round, so that the eight lanes of a row
      // write into eight different groups of banks, and so do those of odd rows, so that two rows read from different ones.
      const int hi = c >> 2, turn = hi ^ (r0 & 1), ka = ((2 * c) & 7) + turn, kb = ((2 * c) & 7) + 1 - turn;
      uint2 xa[8], xb[8];
      const uint8_t *src = ringV + slot * T8_BLK + r0 * 128 + ((c ^ (r0 & 7)) << 4);
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        xa[it] = *reinterpret_cast<const uint2 *>(src + it * 2048 + turn * 8);
        xb[it] = *reinterpret_cast<const uint2 *>(src + it * 2048 + 8 - turn * 8);
      }
      constexpr int TOP = 134 + A8_V_SHIFT;                 // byte of the largest factor
      uint32_t f[8];                                        // 2^(120 + e - shift); one row per lane and a shuffle per row: 102 against 98 us
      int top = 0;
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int byte = vbytes[it * 16 + r0];
        f[it] = byte == 255 ? 0u : t8_pow2x2(min(byte, TOP) - TOP + 127);
        top = max(top, byte == 255 ? 0 : byte);
      }
      // Rows whose factor is out of range take two steps.  Nothing ends as infinity, whatever the byte (a slot that nobody may
      // see can hold any), which must not meet a weight of 0.
      const bool rare = __any_sync(0xffffffffu, top > TOP);
      __syncwarp();
      if (!rare && lane == 0) mbar_arrive(smem_u32(&vempty[slot]));      // all of it is in registers
      const int wb = li % NW;
      if (li >= NW && !mbar_wait_warp(&wempty[wb], (uint32_t)(li / NW - 1) & 1u, abort_flag, wait_limit, lane)) break;
      uint8_t *dst = sW + wb * 2 * T8_BLK + hi * T8_BLK + r0 * 128;
      uint8_t *da = dst + ((ka ^ (r0 & 7)) << 4), *db = dst + ((kb ^ (r0 & 7)) << 4);
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        uint4 a, b;
        t8_widen4(xa[it].x, f[it], a.x, a.y);
        t8_widen4(xa[it].y, f[it], a.z, a.w);
        t8_widen4(xb[it].x, f[it], b.x, b.y);
        t8_widen4(xb[it].y, f[it], b.z, b.w);
        *reinterpret_cast<uint4 *>(da + it * 2048) = a;
        *reinterpret_cast<uint4 *>(db + it * 2048) = b;
      }
      if (rare) {
#pragma unroll 1
        for (int it = 0; it < 8; ++it) {
          const int byte = vbytes[it * 16 + r0];
          const uint32_t g2 = t8_pow2x2(byte > TOP && byte != 255 ? byte - TOP : 0);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint4 *at = reinterpret_cast<uint4 *>((k ? db : da) + it * 2048);
            uint4 v = *at;
            v.x = t8_mulx2(v.x, g2); v.y = t8_mulx2(v.y, g2);
            v.z = t8_mulx2(v.z, g2); v.w = t8_mulx2(v.w, g2);
            *at = v;
          }
        }
      }
      fence_async_smem();
      __syncwarp();
      if (rare && lane == 0) mbar_arrive(smem_u32(&vempty[slot]));
      if (lane == 0) mbar_arrive(smem_u32(&wfull[wb]));
    }
  } else {
    // ---- softmax: group g takes half g of every block; a thread owns query (TMEM lane) i --------------------------------
    t8_setreg_inc<128>();       // 56 + 2 x 128 + 2 x 80 <= 5 x 96, what the block was launched with
    const int g = (warp - 4) >> 2, w = warp & 3, i = w * 32 + lane;
    const int copy = i / QT, query = i % QT;
    const int k0 = copy * (64 / COPIES);                     // this copy's slots within the group's half of a block
    const uint32_t lane_base = tmem + ((uint32_t)(w * 32) << 16), o_col = lane_base + T8_O_COL + (uint32_t)g * 128u;
    A8Seg s = a8_seek<PRE>(p, pl, ls, slab, g0);
    int item = 0;
    bool ok = true;
    float m = T8_NONE, factor = 0.f;
    uint64_t mask = 0;
    f32x2 l2 = 0ull;
#pragma unroll 1
    for (int li = 0; li < nblk; ++li) {
      const int x = g0 + li;
      if (x == s.x1) { s = a8_seek<PRE>(p, pl, ls, slab, x); ++item; }
      const bool first = li == 0 || x == s.x0, last = li == nblk - 1 || x + 1 == s.x1;
      const bool work = (w * 32) % QT < s.cols;              // some thread of this warp has a query
      const int e = li % T8_NC, b = li & 1;
      const uint32_t s_col = lane_base + (uint32_t)(g * 128 + b * 64);
      ok = mbar_wait_warp(&sfull[g * 2 + b], (uint32_t)(li >> 1) & 1u, abort_flag, wait_limit, lane);
      if (!ok) break;
      if (work) {
        tc_fence_after();
        if (first) {
          m = T8_NONE;
          l2 = 0ull;
          factor = qf[(item % T8_NC) * 128 + i];
          if (!PRE) mask = p.row_mask ? p.row_mask[s.r0 + (s.tile * QT + min(query, s.cols - 1)) / p.G] : ~0ull;
        }
        const int slot0 = s.first + (x - s.x0) * 128;
        const bool whole = slot0 >= s.lo && slot0 + 128 <= s.len;
        const int mine = slot0 + g * 64 + k0;
        const ulonglong2 *kb = reinterpret_cast<const ulonglong2 *>(ks_sh + e * 128 + g * 64 + k0);
        const f32x2 f2 = t8_pack(factor, factor);
        // Scores in base 2, less the reference; -inf where a slot is not seen.  All of them at once: one wait for tensor
        // memory and one vote per block (in chunks of 32, each with its own, two warps per scheduler could not hide them).
        float t[CH];
        t8_ld(s_col + (uint32_t)k0, t);
        const bool none = m == T8_NONE;
        const float ref = none ? 0.f : m;
        const f32x2 r2 = t8_pack(-ref, -ref);
#pragma unroll
        for (int j = 0; j < CH; j += 4) {
          const ulonglong2 k = kb[j >> 2];
          const f32x2 ta = t8_pack(t[j], t[j + 1]), tb = t8_pack(t[j + 2], t[j + 3]);
          t8_unpack(FACTORS_FIRST ? t8_fma2(ta, t8_mul2(k.x, f2), r2) : t8_fma2(t8_mul2(ta, k.x), f2, r2), t[j], t[j + 1]);
          t8_unpack(FACTORS_FIRST ? t8_fma2(tb, t8_mul2(k.y, f2), r2) : t8_fma2(t8_mul2(tb, k.y), f2, r2), t[j + 2], t[j + 3]);
        }
        if (!whole) {
#pragma unroll
          for (int j0 = 0; j0 < CH; j0 += 32) {
            const uint32_t seen = a8_visible<PRE>(s, mask, mine + j0, CH < 32 ? CH : 32);
#pragma unroll
            for (int j = 0; j < (CH < 32 ? CH : 32); ++j)
              if (!((seen >> j) & 1u)) t[j0 + j] = -INFINITY;
          }
        }
        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < CH; j += 2) tops[(j >> 1) & 3] = t8_max3(tops[(j >> 1) & 3], t[j], t[j + 1]);
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        if (__any_sync(0xffffffffu, top > (none ? T8_NONE : T8_SLACK))) {
          // ---- the reference moves to the largest (from none: in a segment's first block; else rarely); what has been summed
          // and weighted follows
          const bool moves = top > (none ? T8_NONE : T8_SLACK);
          if (moves) m = ref + top;
          const float corr = !moves ? 1.f : none ? 0.f : t8_ex2(ref - m);
          l2 = t8_mul2(l2, t8_pack(corr, corr));
          if (!first) {
            // O is at rest once the group's product before has completed
            ok = mbar_wait_warp(&pvdone[g * 2 + (b ^ 1)], (uint32_t)((li - 1) >> 1) & 1u, abort_flag, wait_limit, lane);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
              float v[16];
              tc_ld16(o_col + (uint32_t)k * 16u, v);
#pragma unroll
              for (int j = 0; j < 16; ++j) v[j] *= corr;
              tc_st16(o_col + (uint32_t)k * 16u, v);
            }
          }
          const float by = moves ? m - ref : 0.f;
#pragma unroll
          for (int j = 0; j < CH; ++j) t[j] -= by;
        }
        // weights (below 2^T8_SLACK), their sum, bf16 in place of the scores that have been read
        f32x2 sum[2] = {0ull, 0ull};
        constexpr int CS = CH < 32 ? CH : 32;
#pragma unroll
        for (int j0 = 0; j0 < CH; j0 += CS) {
          uint32_t u[CS / 2];
#pragma unroll
          for (int j = 0; j < CS; j += 2) {
            const float a = t8_ex2(t[j0 + j]), d = t8_ex2(t[j0 + j + 1]);
            sum[(j >> 1) & 1] = t8_add2(sum[(j >> 1) & 1], t8_pack(a, d));
            const __nv_bfloat162 z = __floats2bfloat162_rn(a, d);
            u[j >> 1] = *reinterpret_cast<const uint32_t *>(&z);
          }
          t8_st(s_col + (uint32_t)((k0 + j0) / 2), u);
        }
        l2 = t8_add2(l2, t8_add2(sum[0], sum[1]));
        if constexpr (COPIES > 1) {                          // the slots of the other copies
          uint32_t zero[CH / 2];
#pragma unroll
          for (int j = 0; j < CH / 2; ++j) zero[j] = 0u;
#pragma unroll
          for (int k = 0; k < COPIES; ++k)
            if (k != copy) t8_st(s_col + (uint32_t)(k * (CH / 2)), zero);
        }
        tc_wait_st();
        tc_fence_before();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&pfull[g * 2 + b]));
      if (last) {
        // ---- leave the segment: both groups' results become this copy's partial result, half of the columns each ------------
        ok = mbar_wait_warp(&pvdone[g * 2 + b], (uint32_t)(li >> 1) & 1u, abort_flag, wait_limit, lane);
        if (!ok) break;
        float la, lb;
        t8_unpack(l2, la, lb);
        ml_sh[g * 128 + i] = make_float2(m, la + lb);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(xfull));
        ok = mbar_wait_warp(xfull, (uint32_t)item & 1u, abort_flag, wait_limit, lane);
        if (!ok) break;
        if (work) {
          const int64_t row = s.base + (int64_t)QT * blockIdx.x + (int64_t)copy * ls.half + query;
          tc_fence_after();
          const float2 r0 = ml_sh[i], r1 = ml_sh[128 + i];
          const float top = fmaxf(r0.x, r1.x), w0 = t8_ex2(r0.x - top), w1 = t8_ex2(r1.x - top);
          if (g == 0 && query < s.cols) ls.ml[row] = make_float2(top, r0.y * w0 + r1.y * w1);
#pragma unroll 1
          for (int c = g * 2; c < g * 2 + 2; ++c) {
            // 32 columns of 32 rows; eight lanes swap pieces of 16 bytes until each holds the same piece of eight rows, so that
            // a store instruction writes four whole lines (a row per lane, 16 bytes of 32 lines at a time, took 4.5 us)
            float v[32], u[32];
            t8_ld(lane_base + T8_O_COL + (uint32_t)c * 32u, u);
            t8_ld(lane_base + T8_O_COL + 128u + (uint32_t)c * 32u, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = u[j] * w0 + v[j] * w1;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) {
              const bool up = (lane & o) != 0;
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                if (k & o) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const float give = up ? v[k * 4 + j] : v[(k + o) * 4 + j];
                  const float got = __shfl_xor_sync(0xffffffffu, give, o);
                  if (up) v[k * 4 + j] = got; else v[(k + o) * 4 + j] = got;
                }
              }
            }
            // piece lane % 8 of rows (lane / 8) * 8 + k
            float *o = ls.o + (row - (lane & 7)) * 128 + c * 32 + (lane & 7) * 4;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (query - (lane & 7) + k < s.cols)
                *reinterpret_cast<float4 *>(o + k * 128) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
          }
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) { mbar_arrive(smem_u32(&ofree[0])); mbar_arrive(smem_u32(&ofree[1])); }
      }
    }
  }
  tc_teardown(abort_flag, p.status, tmem, 512);
  a8_leave<PRE>(p);
}

// ---- host side -------------------------------------------------------------------------------------------------------
static int t8_slab(int page) { return page % 128 == 0 ? 128 : page % 64 == 0 ? 64 : page % 32 == 0 ? 32 : 16; }
static size_t t8_smem(const SxA8 &p) { return T8_FIXED + a8_plan_bytes(p.B, p.n_groups); }

bool sx_attn8_tc_supported(const SxA8 &p) {
  return p.d == 128 && (int64_t)p.num_pages * p.nkv * p.page < (1ll << 31) - 256 && t8_smem(p) <= T8_SMEM_MAX;
}

template <bool PRE, int COPIES>
static sx_status launch_tc(const SxA8 &p, int sm_count, cudaStream_t st) {
  const int slab = t8_slab(p.page);
  const long long rows = (long long)p.num_pages * p.nkv * p.page;
  CUtensorMap mk, mv;
  if (!sx_tma_map_bytes(p.k, rows, 128, slab, &mk) || !sx_tma_map_bytes(p.v, rows, 128, slab, &mv)) return SX_ERR_CUDA;
  const size_t smem = t8_smem(p);
  // the same value whatever the batch: another thread's call may come between this and the launch
  SX_TRY(sx_rc(cudaFuncSetAttribute(sx_attn8_tc_kernel<PRE, COPIES>, cudaFuncAttributeMaxDynamicSharedMemorySize, T8_SMEM_MAX)));
  return sx_rc(sx_launch(sx_attn8_tc_kernel<PRE, COPIES>, dim3(sm_count), dim3(T8_THREADS), smem, st, mk, mv, p, slab, T8_WAIT_POLLS));
}

sx_status sx_launch_attn8_tc(const SxA8 &p, bool prefix, int sm_count, cudaStream_t st) {
  switch ((prefix ? p.pre : p.own).qt) {
    case 32: return prefix ? launch_tc<true, 4>(p, sm_count, st) : launch_tc<false, 4>(p, sm_count, st);
    case 64: return prefix ? launch_tc<true, 2>(p, sm_count, st) : launch_tc<false, 2>(p, sm_count, st);
    default: return prefix ? launch_tc<true, 1>(p, sm_count, st) : launch_tc<false, 1>(p, sm_count, st);
  }
}
