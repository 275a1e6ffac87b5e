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

struct ScoreSum {
  float m, s, t;
  __device__ __forceinline__ void clear() { m = -INFINITY; s = t = 0.f; }
  // a new reference; sums of nothing have none
  __device__ __forceinline__ void raise(float to, float scale) {
    if (m > -INFINITY) {
      const float d = fmaxf((m - to) * scale, -200.f), f = score_exp2(d);
      t = f * fmaf(s, d, t);
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ void join(float om, float os, float ot, float scale) {
    if (os == 0.f) return;
    if (om > m) raise(om, scale);
    if (om == m || !(om > -INFINITY)) { s += os; t += ot; return; }         // equal references, or a NaN without one
    const float d = fmaxf((om - m) * scale, -200.f), f = score_exp2(d);
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

// Two more elements.  Nothing below 2^-126 of the reference counts; holding d to -200 keeps 0 * -inf out of t.
__device__ __forceinline__ float2 score_add2(float2 a, float2 b) {
  float2 y;
  asm("{.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tadd.rn.f32x2 r, p, q;\n\tmov.b64 {%0, %1}, r;}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}
__device__ __forceinline__ float2 score_mul2(float2 a, float2 b) {
  float2 y;
  asm("{.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmul.rn.f32x2 r, p, q;\n\tmov.b64 {%0, %1}, r;}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}
__device__ __forceinline__ float2 score_fma2(float2 a, float2 b, float2 c) {
  float2 y;
  asm("{.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%6, %7};\n\tfma.rn.f32x2 r, p, q, r;\n\tmov.b64 {%0, %1}, r;}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return y;
}
__device__ __forceinline__ void score_pair(float2 x, float scale, float ref, float2 &s, float2 &t) {
  float2 d = score_mul2(score_add2(x, make_float2(-ref, -ref)), make_float2(scale, scale));
  d = make_float2(score_max_nan(d.x, -200.f), score_max_nan(d.y, -200.f));
  const float2 e = make_float2(score_exp2(d.x), score_exp2(d.y));
  s = score_add2(s, e);
  t = score_fma2(e, d, t);
}
