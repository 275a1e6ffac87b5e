// Decode attention over the 8-bit paged KV cache: the warp-level kernel, the merge of partial results and the
// choice between the warp-level and the tensor-memory kernel (sx_attn8_tc.cu).
//
//   o_r = sum_s w_rs V_s / sum_s w_rs,   w_rs = exp(scale * q_r . K_s),   over the slots s that row r sees
//   K_s = kc_s 2^(ek_s), V_s = vc_s 2^(ev_s)    (e4m3 codes, one exponent per slot and KV head)
//
// The warp-level kernel: a warp streams its run of 16-slot steps (sx_attn8.cuh) through a ring of its own in shared
// memory - cp.async, 512 contiguous bytes per instruction, XOR-swizzled - and needs no other warp.  Both products
// run as mma.sync with the slots (then the head dimension) on the 16-row side and 8 queries on the 8-column side:
//     S^T[slot][q] = sum_d kc[slot][d] Q[q][d]         8-bit, m16n8k32; Q as the sum of an e4m3 and an e5m2 number (a8_split)
//     O^T[d][q] += sum_slot vc[slot][d] P[slot][q]     fp16 x fp16, m16n8k16; e4m3 codes are exact in fp16
// K's fragments are the codes as ldmatrix delivers them.  For V ldmatrix.trans delivers [slot][pair of d]; one byte permute
// splits the pair into two rows of the product, whose order is undone where O is stored, and cvt.f16x2.e4m3x2
// widens them.  The scale of K is a factor of the slot's scores, that of V is added to the score - but a row of V whose
// codes are all zero has weight and gives nothing, so it must not lift the reference that the others' fp16 weights are
// relative to (a sink whose value is zero, 10 nats above the rest, left 5 % of them).  Where such a row would, it is held
// back by A8_ZERO, and what exceeds the range of a weight goes into the sum alone, which is fp32.  Rows are looked at only
// where a reference would move, so the stream pays nothing for it.
//
// Bound by bytes: 12 warps per SM with 12 KB each on their way.  32 sequences of about 4100 slots, 8 heads of 128, one row
// of four queries per head: 263 MB in 53 us of the kernel, 5.0 TB/s with its start and the spread of its ends, about 7 TB/s
// between them, at 55 % of the issue slots; with the merge 57 us.
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>

#include "sx_attn8.cuh"
#include "sx_kernels.cuh"
#include "sx_launch.cuh"

#define A8S_WARPS 4
// How far below its score (in powers of two) a row of zeros puts the reference: the others keep their bits unless they lie
// further below it than this and A8_SLACK together, and its share of the sum, 2^(A8_ZERO + A8_SLACK) at most, leaves room for
// 2^23 such rows in fp32.
#define A8_ZERO 90.f

__device__ __forceinline__ float a8_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void a8_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t a8_transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// e4m3 x e4m3 -> fp32, 16 x 8 x 32; the same with B in e5m2
__device__ __forceinline__ void a8_mma_f8(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void a8_mma_f8_low(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e5m2.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two codes (low half, high half of the register) to fp16 pairs
__device__ __forceinline__ void a8_widen(uint32_t x, uint32_t &lo, uint32_t &hi) {
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(x));
}
// the codes of slots that no query may see can be anything; a code that is not a number must not meet a weight of 0
__device__ __forceinline__ uint32_t a8_finite(uint32_t x) {
  const __half2 top = __float2half2_rn(448.f);
  __half2 v = __hmin2(*reinterpret_cast<__half2 *>(&x), top);
  return *reinterpret_cast<uint32_t *>(&v);
}
__device__ __forceinline__ void a8_cp16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// reads nothing and writes zeros when !valid
__device__ __forceinline__ void a8_cp16_if(uint32_t dst, const void *src, bool valid) {
  const uint32_t bytes = valid ? 16u : 0u;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void a8_cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void a8_cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void a8_ldm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void a8_ldm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Rows of a staged block of 16 that hold nothing but zeros of either sign, as bits; the first codes of a row nearly always
// answer it
template <int D>
__device__ __forceinline__ uint32_t a8_zero_rows(const uint8_t *block, int lane) {
  const uint32_t *row = reinterpret_cast<const uint32_t *>(block + (lane & 15) * D);
  uint32_t zero = __ballot_sync(0xffffffffu, (row[0] & 0x7f7f7f7fu) == 0);
  if (zero) {
    uint32_t any = 0;
#pragma unroll 1
    for (int i = 0; i < D / 4; i += 4) {
      const uint4 x = *reinterpret_cast<const uint4 *>(row + i);
      any |= x.x | x.y | x.z | x.w;
    }
    zero = __ballot_sync(0xffffffffu, (any & 0x7f7f7f7fu) == 0);
  }
  return zero;
}
// 16-byte chunk position of a staged row (D bytes), so that eight rows of an ldmatrix phase fall into different banks
template <int D>
__device__ __forceinline__ int a8_swz(int row, int c) { return c ^ (D >= 128 ? (row & 7) : ((row >> 1) & 3)); }

template <int D, int NQT> struct A8S {
  static constexpr int CTAS = 3;                         // per SM: 12 warps with rings of 16 KB each
  static constexpr int STAGES = D == 128 ? 4 : 8;
  static constexpr int BLK = 16 * D;                     // bytes of the K (or V) codes of a step
  static constexpr int WARP_BYTES = STAGES * 2 * BLK;
  static constexpr int CODES = A8S_WARPS * WARP_BYTES;
  static constexpr int SCALES = A8S_WARPS * STAGES * 32;
};

template <bool PRE, int D, int NQT>
__global__ void __launch_bounds__(A8S_WARPS * 32, (A8S<D, NQT>::CTAS)) sx_attn8_split_kernel(const __grid_constant__ SxA8 p) {
  using C = A8S<D, NQT>;
  constexpr int ST = C::STAGES, BLK = C::BLK, CPR = D / 16;
  extern __shared__ __align__(16) uint8_t a8_smem[];
  a8_enter<PRE>(p);
  const SxA8List &ls = PRE ? p.pre : p.own;
  A8Plan pl;
  a8_plan<PRE, A8S_WARPS * 32>(p, ls, A8_SPLIT_STEP, a8_smem + C::CODES + C::SCALES, pl);
  a8_planned<PRE>(p);
  a8_publish<PRE, A8S_WARPS * 32>(p, pl, ls);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int run = blockIdx.x * A8S_WARPS + warp;
  const int total = pl.cum[pl.units], xb = (int)min((int64_t)total, (int64_t)run * pl.per), xe = min(total - xb, pl.per) + xb;
  if (xb >= xe) { a8_leave<PRE>(p); return; }
  const uint32_t codes = (uint32_t)__cvta_generic_to_shared(a8_smem) + warp * C::WARP_BYTES;
  uint8_t *scale_sh = a8_smem + C::CODES + warp * ST * 32;
  const uint32_t scales = (uint32_t)__cvta_generic_to_shared(scale_sh);

  // ---- loader: requests the step at list position lx into ring stage `st` ---------------------------------
  int lx = xb, l_x1 = xb, l_left = 0, l_off = 0, l_lp = 0, l_h = 0, l_pp = -1;      // slots left in the segment, place in the page
  const int32_t *l_table = p.page_table;
  bool bad = false;
  auto page_at = [&](int lp) -> int { return lp < p.max_pages ? l_table[lp] : -1; };
  // where this lane's 16-byte pieces of a block of codes go; its source is 16 bytes of every 512
  uint32_t at[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int e = i * 32 + lane, row = e / CPR, c = e - row * CPR;
    at[i] = (uint32_t)(row * D + a8_swz<D>(row, c) * 16);
  }
  auto request = [&](int st) {
    if (lx < xe) {
      if (lx == l_x1) {
        const A8Seg s = a8_seek<PRE>(p, pl, ls, A8_SPLIT_STEP, lx);
        const int slot = s.first + (lx - s.x0) * 16;
        l_x1 = s.x1; l_left = s.end - slot; l_h = s.h;
        l_table = p.page_table + (int64_t)s.b0 * p.max_pages;
        l_lp = slot / p.page; l_off = slot - l_lp * p.page;
        l_pp = page_at(l_lp);
      }
      const bool ok = l_pp >= 0 && l_pp < p.num_pages;
      const int64_t row0 = ok ? ((int64_t)l_pp * p.nkv + l_h) * p.page + l_off : 0;
      const uint32_t dst = codes + st * 2 * BLK;
      const uint8_t *kp = p.k + row0 * D + lane * 16, *vp = p.v + row0 * D + lane * 16;
      if (ok && l_left >= 16) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          a8_cp16(dst + at[i], kp + i * 512);
          a8_cp16(dst + BLK + at[i], vp + i * 512);
        }
      } else {                                           // the last slots of a sequence (or no page): zeros behind them
        bad |= !ok;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const bool on = ok && (i * 32 + lane) / CPR < l_left;
          a8_cp16_if(dst + at[i], on ? kp + i * 512 : p.k, on);
          a8_cp16_if(dst + BLK + at[i], on ? vp + i * 512 : p.v, on);
        }
      }
      if (lane < 2) {
        if (ok) a8_cp16(scales + st * 32 + lane * 16, (lane ? p.vs : p.ks) + row0);
        else *reinterpret_cast<uint4 *>(scale_sh + st * 32 + lane * 16) = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
      }
      ++lx;
      l_left -= 16;
      l_off += 16;
      if (l_off == p.page && lx < l_x1) { l_off = 0; l_pp = page_at(++l_lp); }       // needed a step later
    }
    a8_cp_commit();
  };
#pragma unroll 1
  for (int i = 0; i < ST - 1; ++i) request(i);

  A8Seg seg;
  seg.x1 = xb;
  uint32_t qf[NQT][CPR][2];
  float qs[NQT][2], M[NQT][2], L[NQT][2], O[NQT][CPR][4];
  uint64_t vis[NQT][2];
  int st = 0;
#pragma unroll 1
  for (int x = xb; x < xe; ++x) {
    if (x == seg.x1) {
      // ---- a new (unit, head, tile): its queries in two 8-bit parts --------------------------------------------
      seg = a8_seek<PRE>(p, pl, ls, A8_SPLIT_STEP, x);
#pragma unroll
      for (int i = 0; i < NQT; ++i) {
        const int col = i * 8 + g, qi = seg.tile * ls.qt + col, j = qi / p.G;
        const bool live = col < seg.cols;
        const bf16 *src = p.q + (int64_t)(seg.r0 + j) * p.q_stride + (int64_t)(seg.h * p.G + qi - j * p.G) * D + t * 4;
        uint2 raw[CPR];
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < CPR; ++c) {
          raw[c] = live ? *reinterpret_cast<const uint2 *>(src + c * 16) : make_uint2(0, 0);
          top = __vmaxu2(top, __vmaxu2(raw[c].x & 0x7fff7fffu, raw[c].y & 0x7fff7fffu));
        }
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^-ex brings the largest magnitude into (224, 448]
        const int te = (int)(top >> 7);
        const int ex = te == 0 || te == 255 ? 0 : max(-126, te - 135 + ((top & 0x7f) > 96 ? 1 : 0));
        const float up = __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
        for (int c = 0; c < CPR; ++c) {
          uint32_t hi = 0, lo = 0;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t w = k ? raw[c].y : raw[c].x;
            const float2 f = make_float2(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
            uint32_t h2, l2;
            a8_split(f, te != 255, h2, l2);
            hi |= h2 << (16 * k);
            lo |= l2 << (16 * k);
          }
          qf[i][c][0] = hi;
          qf[i][c][1] = lo;
        }
        const float mine = __uint_as_float((uint32_t)(127 + ex) << 23) * p.scale_log2;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          qs[i][k] = __shfl_sync(0xffffffffu, mine, (2 * t + k) * 4);
          M[i][k] = -INFINITY;
          L[i][k] = 0.f;
          if (!PRE) {
            const int cq = i * 8 + 2 * t + k, qq = seg.tile * ls.qt + min(cq, seg.cols - 1);
            vis[i][k] = p.row_mask ? p.row_mask[seg.r0 + qq / p.G] : ~0ull;
          }
        }
#pragma unroll
        for (int c = 0; c < CPR; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) O[i][c][k] = 0.f;
      }
    }
    a8_cp_wait<ST - 2>();
    __syncwarp();
    request((st + ST - 1) % ST);               // the stage of the step before, which every lane has left
    const int slot0 = seg.first + (x - seg.x0) * 16;
    const bool whole = PRE ? slot0 + 16 <= seg.end : (slot0 >= seg.lo && slot0 + 16 <= seg.len);
    const uint32_t kb = codes + st * 2 * BLK, vb = kb + BLK;
    const uint8_t *sb = scale_sh + st * 32;
    // ---- S^T: lane (g, t) holds slots g and g + 8, queries 2t and 2t + 1 ---------------------------------------
    float S[NQT][4];
#pragma unroll
    for (int i = 0; i < NQT; ++i) S[i][0] = S[i][1] = S[i][2] = S[i][3] = 0.f;
    const int lrow = (lane & 7) + ((lane >> 3) & 1) * 8, lc = lane >> 4;
#pragma unroll
    for (int c = 0; c < CPR; c += 2) {
      uint32_t r[4];
      a8_ldm4(kb + lrow * D + a8_swz<D>(lrow, c + lc) * 16, r);
#pragma unroll
      for (int i = 0; i < NQT; ++i) {
        a8_mma_f8(S[i], r, qf[i][c][0], qf[i][c + 1][0]);
        a8_mma_f8_low(S[i], r, qf[i][c][1], qf[i][c + 1][1]);
      }
    }
    float kscale[2], ev[2], inv[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int kbyte = sb[g + r * 8], vbyte = sb[16 + g + r * 8];
      kscale[r] = a8_pow2(kbyte);
      ev[r] = a8_exponent(vbyte);
      inv[r] = a8_pow2_inv(vbyte);
    }
    bool up = false;
#pragma unroll
    for (int i = 0; i < NQT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) S[i][k] = fmaf(S[i][k] * qs[i][k & 1], kscale[k >> 1], ev[k >> 1]);
    if (!whole) {
#pragma unroll
      for (int i = 0; i < NQT; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t seen = a8_visible<PRE>(seg, vis[i][k], slot0, 16) >> g;
          if (!(seen & 1u)) S[i][k] = -INFINITY;
          if (!(seen & 256u)) S[i][2 + k] = -INFINITY;
        }
    }
#pragma unroll
    for (int i = 0; i < NQT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) up |= S[i][k] > M[i][k & 1] + A8_SLACK;
    if (__any_sync(0xffffffffu, up)) {
      // a reference moves: it only has to keep the weights in range, so this is rare behind the first steps
      const uint32_t zero = a8_zero_rows<D>(a8_smem + warp * C::WARP_BYTES + st * 2 * BLK + BLK, lane);
      const bool z[2] = {((zero >> g) & 1u) != 0, ((zero >> (g + 8)) & 1u) != 0};
      const float back[2] = {z[0] ? ev[0] + A8_ZERO : 0.f, z[1] ? ev[1] + A8_ZERO : 0.f};
#pragma unroll
      for (int i = 0; i < NQT; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float bm = fmaxf(S[i][k] - back[0], S[i][k + 2] - back[1]);
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, o));
          if (bm > M[i][k] + A8_SLACK) {
            const float w = a8_ex2(M[i][k] - bm);              // 0 for the first one
            M[i][k] = bm;
            L[i][k] *= w;
#pragma unroll
            for (int c = 0; c < CPR; ++c) { O[i][c][k] *= w; O[i][c][k + 2] *= w; }
          }
        }
      if (zero) {
#pragma unroll
        for (int i = 0; i < NQT; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (z[k >> 1] && S[i][k] > M[i][k & 1] + A8_SLACK) {
              L[i][k & 1] += a8_ex2(S[i][k] - ev[k >> 1] - M[i][k & 1]);
              S[i][k] = -INFINITY;
            }
      }
    }
    // ---- weights (below 2^14), their sums without the value scale, P^T as fp16 -----------------------------------
    uint32_t pb[NQT][2];
#pragma unroll
    for (int i = 0; i < NQT; ++i) {
      float w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float m = M[i][k & 1];
        w[k] = a8_ex2(S[i][k] - (m == -INFINITY ? 0.f : m));
        L[i][k & 1] += (!whole && w[k] == 0.f) ? 0.f : w[k] * inv[k >> 1];
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        __half2 h = __floats2half2_rn(w[2 * r], w[2 * r + 1]);
        pb[i][r] = a8_transpose(*reinterpret_cast<uint32_t *>(&h));
      }
    }
    // ---- O^T: rows 2g and 2g + 1 of each 16-row chunk of the head dimension ---------------------------------------
#pragma unroll
    for (int c = 0; c < CPR; c += 2) {
      uint32_t r[4], a[8];
      a8_ldm4t(vb + lrow * D + a8_swz<D>(lrow, c + lc) * 16, r);
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = __byte_perm(r[k], 0, 0x3120);     // slots side by side, per row of d
      a8_widen(r[0], a[0], a[1]);
      a8_widen(r[1], a[2], a[3]);
      a8_widen(r[2], a[4], a[5]);
      a8_widen(r[3], a[6], a[7]);
      if (!whole) {
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = a8_finite(a[k]);
      }
#pragma unroll
      for (int i = 0; i < NQT; ++i) {
        a8_mma(O[i][c], a[0], a[1], a[2], a[3], pb[i][0], pb[i][1]);
        a8_mma(O[i][c + 1], a[4], a[5], a[6], a[7], pb[i][0], pb[i][1]);
      }
    }
    st = (st + 1) % ST;
    if (x + 1 == seg.x1 || x + 1 == xe) {
      // ---- leave the segment: the partial result of this run ------------------------------------------------------
      const int64_t row = seg.base + (int64_t)ls.qt * run;
#pragma unroll
      for (int i = 0; i < NQT; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float l = L[i][k];
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
          const int col = i * 8 + 2 * t + k;
          if (col < seg.cols) {
            if (g == 0) ls.ml[row + col] = make_float2(M[i][k], l);
            float *o = ls.o + (row + col) * D + 2 * g;
#pragma unroll
            for (int c = 0; c < CPR; ++c)
              *reinterpret_cast<float2 *>(o + c * 16) = make_float2(O[i][c][k], O[i][c][k + 2]);
          }
        }
    }
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) sx_set_status(p.status, SX_ERR_CAPACITY);
  a8_leave<PRE>(p);
}

// ---- merge -------------------------------------------------------------------------------------------------------
// o[row, head] = sum over the partial results of 2^(ref - max ref) O, over the same sum of l; zero when no slot is
// seen.  W warps share the partial results of a (row, query head), a lane owns D / 32 columns; a CTA has 8 / W of them.
template <int D, int W>
__global__ void __launch_bounds__(A8_MERGE_THREADS) sx_attn8_merge_kernel(const __grid_constant__ SxA8 p) {
  constexpr int V = D / 32, PER = A8_MERGE_THREADS / 32 / W;
  __shared__ float2 ml_sh[PER][W];
  __shared__ float o_sh[PER][W][D];
  sx_pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % W, mine = warp / W;
  const int64_t at0 = (int64_t)blockIdx.x * PER + mine;
  const bool live = at0 < (int64_t)p.B * p.rows * p.nq;
  const int r = live ? (int)(at0 / p.nq) : 0, hq = live ? (int)(at0 - (int64_t)r * p.nq) : 0, b = r / p.rows, j = r - b * p.rows, h = hq / p.G;
  sx_pdl_wait();
  float M = -INFINITY, L = 0.f, acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  const int gq = hq - h * p.G, grp = p.n_groups > 0 ? p.seq_group[b] : -1;
#pragma unroll 1
  for (int list = 0; list < (grp >= 0 ? 2 : 1); ++list) {
    // the own list, then the prefix list: unit, queries of the unit, which of them, first row of the unit
    const SxA8List &ls = list ? p.pre : p.own;
    const int s = list ? p.group_start[grp] : b, u = list ? grp : b;
    const int nq = (list ? a8_members(p, grp) : 1) * p.rows * p.G, q = ((b - s) * p.rows + j) * p.G + gq;
    const float unit = ls.unit;
    const int steps = ls.steps[u], cum = ls.cum[u];
    const uint32_t per = (uint32_t)a8_per(ls.total[0], ls);
    if (steps == 0) continue;
    const uint32_t x0 = (uint32_t)(cum + (h * a8_tiles(nq, ls.qt_shift) + (q >> ls.qt_shift)) * steps);
    // partial k of this row: part k mod 2^parts_shift of run c0 + k / 2^parts_shift
    const uint32_t c0 = x0 / per;
    const int n = (int)((x0 + (uint32_t)steps - 1u) / per - c0 + 1u) << ls.parts_shift;
    const int64_t base = ((int64_t)s * p.rows * p.nkv) * p.G + (int64_t)h * nq + q + ((int64_t)c0 << ls.qt_shift);
#pragma unroll 1
    for (int k0 = part; k0 < n; k0 += 4 * W) {
      float2 ml[4];
      float v[4][V];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool on = k0 + k * W < n;
        const int kk = on ? k0 + k * W : k0, run = kk >> ls.parts_shift;
        const int64_t at = base + ((int64_t)run << ls.qt_shift) + (kk - (run << ls.parts_shift)) * ls.half;
        ml[k] = ls.ml[at];
        if (!on) ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) v[k][i] = ls.o[at * D + lane * V + i];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (ml[k].x == -INFINITY && ml[k].y == 0.f) continue;         // nothing seen there
        const float m = fmaxf(M, ml[k].x), a = (M == -INFINITY) ? 0.f : a8_ex2(M - m), w = a8_ex2(ml[k].x - m);
        M = m;
        L = L * a + ml[k].y * w;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = acc[i] * a + v[k][i] * (w * unit);
      }
    }
  }
  if (W > 1) {
    if (lane == 0) ml_sh[mine][part] = make_float2(M, L);
#pragma unroll
    for (int i = 0; i < V; ++i) o_sh[mine][part][lane * V + i] = acc[i];
    __syncthreads();
    if (part != 0) return;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, ml_sh[mine][w].x);
    L = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float2 v = ml_sh[mine][w];
      if (v.x == -INFINITY && v.y == 0.f) continue;
      const float f = a8_ex2(v.x - m);
      L += v.y * f;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += o_sh[mine][w][lane * V + i] * f;
    }
  }
  if (!live) return;
  bf16 y[V];
#pragma unroll
  for (int i = 0; i < V; ++i) y[i] = __float2bfloat16_rn(L == 0.f ? 0.f : acc[i] / L * p.unit);
  bf16 *o = p.o_out + ((int64_t)r * p.nq + hq) * D + lane * V;
  if (V == 4) *reinterpret_cast<uint2 *>(o) = *reinterpret_cast<uint2 *>(y);
  else *reinterpret_cast<uint32_t *>(o) = *reinterpret_cast<uint32_t *>(y);
}

// ---- host side -------------------------------------------------------------------------------------------------------
static int split_runs(int sm_count) { return sm_count * 3 * A8S_WARPS; }

template <bool PRE, int D, int NQT>
static sx_status launch_split(const SxA8 &p, int sm_count, cudaStream_t st) {
  using C = A8S<D, NQT>;
  const size_t smem = C::CODES + C::SCALES + a8_plan_bytes(p.B, p.n_groups);
  static_assert(C::CODES + C::SCALES + 48 * 1024 < 200 * 1024, "ring and the largest plan fit one SM");
  // Set on every call: the attribute belongs to the current device, and setting it costs less than remembering it.  Always to
  // the same value, the largest plan's: another thread's call for a smaller batch may come between this and the launch.
  const int most = C::CODES + C::SCALES + (int)a8_plan_bytes(A8_MAX_UNITS, A8_MAX_UNITS);
  SX_TRY(sx_rc(cudaFuncSetAttribute(sx_attn8_split_kernel<PRE, D, NQT>, cudaFuncAttributeMaxDynamicSharedMemorySize, most)));
  SX_TRY(sx_rc(cudaFuncSetAttribute(sx_attn8_split_kernel<PRE, D, NQT>, cudaFuncAttributePreferredSharedMemoryCarveout, 100)));
  return sx_rc(sx_launch(sx_attn8_split_kernel<PRE, D, NQT>, dim3(sm_count * C::CTAS), dim3(A8S_WARPS * 32), smem, st, p));
}

// one list with the warp-level kernel
template <bool PRE>
static sx_status split_list(SxA8 &p, int sm_count, cudaStream_t st) {
  const int qt = (PRE ? p.pre : p.own).qt;
  if (p.d == 128) return qt == 8 ? launch_split<PRE, 128, 1>(p, sm_count, st) : launch_split<PRE, 128, 2>(p, sm_count, st);
  return qt == 8 ? launch_split<PRE, 64, 1>(p, sm_count, st) : launch_split<PRE, 64, 2>(p, sm_count, st);
}

static size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
// Queries per tile of the tensor-memory kernel for `q` per KV head: with 32 (64) the softmax is spread over four
// (two) copies of them, which leave a partial result each (eight prefixes of 4096 slots under 32 queries: 67 us, in a tile
// of 128 for the same 32 71 us); bounded, so that the workspace of a large batch is not four times what it needs.
#define A8_COPY_ROWS 65536
static int tc_tile(int q, size_t all) {
  const int qt = q <= 32 ? 32 : q <= 64 ? 64 : 128;
  return (128 / qt) * all <= A8_COPY_ROWS ? qt : 128;
}
// rows of partial results that any variant of a list may use
static size_t list_rows(int nq, int B, int rows, int sm_count) {
  const size_t q = (size_t)B * rows * nq, split = (size_t)16 * split_runs(sm_count) + q, most = 4 * q < A8_COPY_ROWS ? 4 * q : A8_COPY_ROWS,
               tc = (size_t)128 * sm_count + (most > q ? most : q);
  return split > tc ? split : tc;
}
static size_t list_bytes(int nq, int d, int B, int rows, int units, int sm_count) {
  return 2 * up256((size_t)units * 4) + 256 +
         up256(list_rows(nq, B, rows, sm_count) * 8) + up256(list_rows(nq, B, rows, sm_count) * d * 4);
}

size_t sx_attn8_ws_bytes(int nq, int nkv, int d, int B, int rows, int groups, int sm_count) {
  (void)nkv;
  return up256((size_t)B * 4) + list_bytes(nq, d, B, rows, B, sm_count) +
         (groups > 0 ? list_bytes(nq, d, B, rows, groups, sm_count) : 0);
}

template <int D, int W>
static sx_status launch_merge(const SxA8 &p, cudaStream_t st) {
  const int64_t rows = (int64_t)p.B * p.rows * p.nq, per = A8_MERGE_THREADS / 32 / W;
  SX_TRY(sx_rc(cudaFuncSetAttribute(sx_attn8_merge_kernel<D, W>, cudaFuncAttributePreferredSharedMemoryCarveout, 100)));
  return sx_rc(sx_launch(sx_attn8_merge_kernel<D, W>, dim3((unsigned)((rows + per - 1) / per)), dim3(A8_MERGE_THREADS), 0, st, p));
}
// Warps per output row: as many as fill the SMs about once (a row's partial results are a chain of loads: with one warp per
// row 32 x 4100 slots take 78 us instead of 57 us, 4096 slots 27 us instead of 15 us), one where the rows alone fill them
template <int D>
static sx_status merge(const SxA8 &p, int sm_count, cudaStream_t st) {
  const int64_t rows = (int64_t)p.B * p.rows * p.nq, slots = 8ll * sm_count;       // CTAs of 256 threads at a time
  return rows <= slots / 2 ? launch_merge<D, 8>(p, st) : rows <= 2 * slots ? launch_merge<D, 4>(p, st) : launch_merge<D, 1>(p, st);
}

// Queries per KV head of a unit, in the own list and in the prefix list.
static int own_queries(const SxA8 &p) { return p.rows * p.G; }
// The host knows how many groups there are, not which; it takes them to be alike.  (A larger one becomes several tiles: a
// group of 29 sequences among four of 32 takes 48 us instead of 43 us with the tile that it needs, but sixteen pairs take
// 50 us instead of 87 us with the tile that one large group among them would need; prefixes of 4096 slots.)
static int pre_queries(const SxA8 &p) { return p.n_groups > 0 ? (p.B + p.n_groups - 1) / p.n_groups * own_queries(p) : 0; }
// Which kernel takes a list of `q` queries per KV head.  The warp-level kernel reads a unit's slots once for every 16
// queries and is bound by bytes up to there; the tensor-memory kernel's time per block of slots hardly depends on the queries.
// Up to 16 queries the first is faster (one row of 4 heads over 32 x 4100 slots 57 against 107 us, one row of 8 heads
// over 8 x 16384 slots 63 against 93 us, one of 4096 slots 15 against 27 us), beyond 16 the second (32 queries, 4 x 32768
// slots: 98 against 146 us; a prefix of 16384 slots under 128 queries: 50 against 92 us; 4 prefixes under 128: 93
// against 213 us).
static sx_status choose(const SxA8 &p, int kernel, int q, int sm_count, SxA8List &ls, bool &tc) {
  auto log2i = [](int v) { int s = 0; while ((1 << s) < v) ++s; return s; };
  const bool can = sx_attn8_tc_supported(p);
  if (kernel == SX_ATTN_TC && !can) return SX_ERR_UNSUPPORTED;
  tc = can && (kernel == SX_ATTN_TC || (kernel == SX_ATTN_AUTO && q > 16));
  ls.step = tc ? A8_TC_STEP : A8_SPLIT_STEP;
  ls.qt = tc ? tc_tile(q, (size_t)p.B * p.rows * p.nq) : q <= 8 ? 8 : 16;
  ls.runs = tc ? sm_count : split_runs(sm_count);
  ls.min_per = tc ? 1 : 4;
  ls.spread = sm_count;
  ls.qt_shift = log2i(ls.qt);
  ls.step_shift = log2i(ls.step);
  ls.parts_shift = tc ? log2i(128 / ls.qt) : 0;
  ls.half = (int64_t)ls.qt * sm_count + (int64_t)p.B * p.rows * p.nq;
  // list positions are 32-bit: steps of a sequence's whole capacity x KV heads x tiles of all units
  const int64_t steps = (int64_t)p.max_pages * p.page / ls.step + 2, tiles = (int64_t)p.B * p.rows * p.G / ls.qt + p.B + p.n_groups;
  return steps * p.nkv * tiles < (1ll << 31) - (1 << 20) ? SX_OK : SX_ERR_UNSUPPORTED;
}
static sx_status choose_both(SxA8 &p, int kernel, int sm_count, bool &own_tc, bool &pre_tc) {
  if ((p.d != 64 && p.d != 128) || p.page % A8_SPLIT_STEP || p.B + p.n_groups > A8_MAX_UNITS) return SX_ERR_UNSUPPORTED;
  SX_TRY(choose(p, kernel, own_queries(p), sm_count, p.own, own_tc));
  return p.n_groups > 0 ? choose(p, kernel, pre_queries(p), sm_count, p.pre, pre_tc) : SX_OK;
}
sx_status sx_attn8_check(SxA8 p, int kernel, int sm_count) {
  bool own_tc = false, pre_tc = false;
  return choose_both(p, kernel, sm_count, own_tc, pre_tc);
}

sx_status sx_launch_attn8(SxA8 p, int kernel, char *ws, int sm_count, cudaStream_t st) {
  bool own_tc = false, pre_tc = false;
  SX_TRY(choose_both(p, kernel, sm_count, own_tc, pre_tc));
  size_t o = 0;
  auto take = [&](size_t bytes) { char *at = ws + o; o += up256(bytes); return at; };
  p.seq_group = (int32_t *)take((size_t)p.B * 4);
  auto place = [&](SxA8List &ls, int units) {
    ls.cum = (int32_t *)take((size_t)units * 4);
    ls.steps = (int32_t *)take((size_t)units * 4);
    ls.total = (int32_t *)take(4);
    ls.ml = (float2 *)take(list_rows(p.nq, p.B, p.rows, sm_count) * 8);
    ls.o = (float *)take(list_rows(p.nq, p.B, p.rows, sm_count) * p.d * 4);
  };
  place(p.own, p.B);
  if (p.n_groups > 0) place(p.pre, p.n_groups);
  p.unit = own_tc || pre_tc ? ldexpf(1.f, A8_V_SHIFT) : 1.f;
  p.own.unit = own_tc ? 1.f : 1.f / p.unit;
  p.pre.unit = pre_tc ? 1.f : 1.f / p.unit;
  if (p.n_groups > 0) {
    SX_TRY(pre_tc ? sx_launch_attn8_tc(p, true, sm_count, st) : split_list<true>(p, sm_count, st));
    p.after_prefix = 1;
  }
  SX_TRY(own_tc ? sx_launch_attn8_tc(p, false, sm_count, st) : split_list<false>(p, sm_count, st));
  return p.d == 128 ? merge<128>(p, sm_count, st) : merge<64>(p, sm_count, st);
}
