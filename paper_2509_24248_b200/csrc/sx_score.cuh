// Running softmax sums of rows of logits, shared by the pass over logits in memory (sx_score.cu) and the epilogue of the head's
// product (sx_gemm_tc.cu).
#pragma once
#include "sx_common.cuh"

__device__ __forceinline__ float score_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the larger of two, NaN if either is
__device__ __forceinline__ float score_max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// (a - b) * by, rounded as that is but for differences beyond fp32's range, which halves keep in it (by up to 2^100): logits at both
// ends of it are close together at a high temperature.
__device__ __forceinline__ float score_gap(float a, float b, float by) { return fmaf(a, 0.5f, -0.5f * b) * (2.f * by); }

struct ScoreSum {
  float m, s, t;
  __device__ __forceinline__ void clear() { m = -INFINITY; s = t = 0.f; }
  // a new reference; sums of nothing have none
  __device__ __forceinline__ void raise(float to, float scale) {
    if (m > -INFINITY) {
      const float d = fmaxf(score_gap(m, to, scale), -200.f), f = score_exp2(d);
      t = f * fmaf(s, d, t);
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ void join(float om, float os, float ot, float scale) {
    if (os == 0.f) return;
    if (om > m) raise(om, scale);
    if (om == m || !(om > -INFINITY)) { s += os; t += ot; return; }         // equal references, or a NaN without one
    const float d = fmaxf(score_gap(om, m, scale), -200.f), f = score_exp2(d);
    t += f * fmaf(os, d, ot);
    s = fmaf(os, f, s);
  }
  __device__ __forceinline__ void warp_join(float scale) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o), ot = __shfl_xor_sync(0xffffffffu, t, o);
      join(om, os, ot, scale);
    }
  }
};

// Two more elements.  Nothing below 2^-126 of the reference counts; holding d to -200 keeps 0 * -inf out of t.  (Packed fp32
// pairs were tried: the moves that bring the pairs together cost more than the instructions saved.)
__device__ __forceinline__ void score_pair(float2 x, float scale, float ref, float2 &s, float2 &t) {
  const float d0 = score_max_nan(score_gap(x.x, ref, scale), -200.f), d1 = score_max_nan(score_gap(x.y, ref, scale), -200.f);
  const float e0 = score_exp2(d0), e1 = score_exp2(d1);
  s.x += e0;
  s.y += e1;
  t.x = fmaf(e0, d0, t.x);
  t.y = fmaf(e1, d1, t.y);
}

// Eight floats to a 32-byte boundary, a whole sector.  PASS: hardly any of them will be read again, so they are the first to leave the
// L2 (600 MB of logits beside a product that lives on the L2: 1.01 instead of 1.10-1.15 ms).
template <bool PASS>
__device__ __forceinline__ void sx_store8(float *dst, const float *v) {
  if (PASS)
    asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(dst), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
  else
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(dst), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}
