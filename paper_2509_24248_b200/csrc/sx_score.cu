// Log-probabilities of given tokens, entropy and best alternatives, from rows of logits and from hidden states through a head.
//
// With c = log2(e) / temperature, per row of logits x
//     m = max x,   d = c (x - m),   s = sum 2^d,   t = sum 2^d d
//     log p = (x - m) / temperature - ln s,        entropy = ln 2 (log2 s - t / s)
// in one pass: a lane keeps (m, s, t) of what it has seen and takes a new reference when a group of its elements is above
// the old one.  Sums, references and results are fp32.  The reference is a logit itself and the difference is taken first:
// a rounding of d is relative to d, and a row that holds nothing but its type's lowest value is as good as any other.
//
// Alternatives without a sort: the row is cut into groups of neighbouring elements whose maxima fall out of the pass.  The k
// best elements (larger first, then the lower index) lie in the k best groups (larger maximum first, then the lower group), so
// every warp keeps a sorted list of its 32 best groups, one per lane; the lists are joined by counting, for each entry, how many
// others are before it, and the elements of the k best groups that are not below the k-th of these maxima are ranked the
// same way.  The cost does not depend on the values but for the number of insertions.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "sx_kernels.cuh"
#include "sx_launch.cuh"

namespace cg = cooperative_groups;

#define SCORE_THREADS 256
#define SCORE_WARPS (SCORE_THREADS / 32)
#define SCORE_GROUP_BYTES 64
#define SCORE_MAX_GROUP 32             // elements of a group
#define SCORE_MAX_CLUSTER 8

struct SxScoreArgs {
  int T, V, n_given, top;
  float scale, inverse;                // log2(e) / temperature, 1 / temperature
  const int32_t *tok;
  float *logp, *entropy, *top_logp;
  int32_t *top_tok, *status;
};

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

// The 32 best (value, id) that a warp has met, best first, lane by lane.  Entries come with ascending ids, so an equal value goes
// behind.
struct ScoreList {
  float v;
  int id;
  __device__ __forceinline__ void clear() { v = -INFINITY; id = -1; }
  __device__ __forceinline__ void insert(float nv, int nid, int lane) {
    // an entry stays in front if it is not smaller; empty ones (id -1) are behind everything
    const int at = __popc(__ballot_sync(0xffffffffu, id >= 0 && v >= nv));
    const float uv = __shfl_up_sync(0xffffffffu, v, 1);
    const int ui = __shfl_up_sync(0xffffffffu, id, 1);
    if (lane > at) { v = uv; id = ui; }
    if (lane == at) { v = nv; id = nid; }
  }
  // a candidate of every lane, ids ascending with the lanes; those that cannot be among the first `top` are left out
  __device__ __forceinline__ void offer(float nv, int nid, bool on, int top, int lane) {
    const float kth = __shfl_sync(0xffffffffu, v, top - 1);
    const int kid = __shfl_sync(0xffffffffu, id, top - 1);
    uint32_t m = __ballot_sync(0xffffffffu, on && (kid < 0 || nv > kth));
    while (m) {
      const int l = __ffs(m) - 1;
      m &= m - 1;
      insert(__shfl_sync(0xffffffffu, nv, l), __shfl_sync(0xffffffffu, nid, l), lane);
    }
  }
};

struct ScoreShared {
  unsigned long long list[SCORE_WARPS * 32];                          // the warps' lists of groups, packed (value, id)
  unsigned long long group[32];                                       // the best groups
  unsigned long long cand[32 * SCORE_MAX_GROUP];                      // their elements that can be among the best
  unsigned long long best[SCORE_MAX_CLUSTER * 32];                    // the best elements (of every CTA of a row, in the first)
  float sum[SCORE_WARPS][3], row[3];
  int n_cand;
};

// ---- steps shared by both forms; every thread of the CTA calls them ------------------------------------------------
// sums of the warps -> sh.row
__device__ __forceinline__ void score_block_sum(ScoreShared &sh, ScoreSum a, float scale) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  a.warp_join(scale);
  if (lane == 0) { sh.sum[warp][0] = a.m; sh.sum[warp][1] = a.s; sh.sum[warp][2] = a.t; }
  __syncthreads();
  if (warp == 0) {
    ScoreSum b;
    b.clear();
    if (lane < SCORE_WARPS) { b.m = sh.sum[lane][0]; b.s = sh.sum[lane][1]; b.t = sh.sum[lane][2]; }
    b.warp_join(scale);
    if (lane == 0) { sh.row[0] = b.m; sh.row[1] = b.s; sh.row[2] = b.t; }
  }
  __syncthreads();
}

// the warps' lists -> the `top` best groups in sh.group (0: none)
__device__ __forceinline__ void score_best_groups(ScoreShared &sh, const ScoreList &l, int top) {
  const int lane = threadIdx.x & 31;
  const unsigned long long mine = l.id >= 0 ? sx_pack(l.v, (uint32_t)l.id) : 0ull;
  sh.list[threadIdx.x] = mine;
  if (threadIdx.x < 32) sh.group[threadIdx.x] = 0ull;
  if (threadIdx.x == 0) sh.n_cand = 0;
  __syncthreads();
  if (mine && lane < top) {
    int rank = 0;
    for (int w = 0; w < SCORE_WARPS; ++w) {
      // lists descend: the number of entries before mine, by halving
      const unsigned long long *p = sh.list + w * 32;
      int lo = 0;
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
        if (p[lo + step - 1] > mine) lo += step;
      rank += lo + (p[lo] > mine ? 1 : 0);
    }
    if (rank < top) sh.group[rank] = mine;
  }
  __syncthreads();
}

// one element of one of the best groups
__device__ __forceinline__ void score_candidate(ScoreShared &sh, float v, int index, float kth) {
  if (v >= kth && v > -INFINITY) sh.cand[atomicAdd(&sh.n_cand, 1)] = sx_pack(v + 0.f, (uint32_t)index);    // -0 counts as 0
}

// The `top` best of n different keys in src, best first, to dst (0 behind the last).  The order in which src was filled does not
// matter.
__device__ __forceinline__ void score_rank(const unsigned long long *src, int n, int top, unsigned long long *dst) {
  for (int i = threadIdx.x; i < top; i += SCORE_THREADS)
    if (i >= n) dst[i] = 0ull;
  for (int i = threadIdx.x; i < n; i += SCORE_THREADS) {
    const unsigned long long mine = src[i];
    int rank = mine ? 0 : top;
    for (int j = 0; j < n && rank < top; ++j) rank += src[j] > mine ? 1 : 0;
    if (mine && rank < top) dst[rank] = mine;
  }
}

// Results of a row.  logit(i): the raw logit of token i.  A row with a NaN or an infinite logit has no probabilities: NaN, and no
// alternatives; where every logit is -inf no token has any.
template <typename F>
__device__ __forceinline__ void score_write(const ScoreShared &sh, const SxScoreArgs &p, int row, const unsigned long long *best, F logit) {
  const float m = sh.row[0], s = sh.row[1], t = sh.row[2], LN2 = 0.6931471805599453f, NaN = __int_as_float(0x7fffffff);
  const bool bad = !(s >= 0.f) || m == INFINITY, none = !bad && m == -INFINITY;
  const float ln = none ? 0.f : logf(s);
  const auto log_p = [&](float x) { return fmaf(x - m, p.inverse, -ln); };
  for (int i = threadIdx.x; i < p.n_given; i += SCORE_THREADS) {
    const int64_t at = (int64_t)row * p.n_given + i;
    const int tok = p.tok[at];
    float y = 0.f;
    if (tok >= 0 && tok < p.V) {
      const float x = logit(tok);
      y = bad ? NaN : x == -INFINITY ? -INFINITY : log_p(x);
    } else if (tok != -1) {
      y = NaN;
      sx_set_status(p.status, SX_ERR_CAPACITY);
    }
    p.logp[at] = y;
  }
  if (p.entropy && threadIdx.x == 0) p.entropy[row] = bad ? NaN : none ? 0.f : ln - LN2 * (t / s);
  for (int i = threadIdx.x; i < p.top; i += SCORE_THREADS) {
    const unsigned long long key = best[i];
    const int64_t at = (int64_t)row * p.top + i;
    const bool on = key != 0ull && !bad;
    if (p.top_tok) p.top_tok[at] = on ? (int)sx_pack_index(key) : -1;
    if (p.top_logp) p.top_logp[at] = bad ? NaN : on ? log_p(sx_pack_value(key)) : -INFINITY;
  }
}

// ---- rows of logits ------------------------------------------------------------------------------------------------------
template <typename E> struct ScoreElem;
template <> struct ScoreElem<bf16> {
  static __device__ __forceinline__ float one(bf16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ void pair(uint32_t w, float *a, float *b) { *a = __uint_as_float(w << 16); *b = __uint_as_float(w & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) {
    const __nv_bfloat162 y = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&y);
  }
};
template <> struct ScoreElem<__half> {
  static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
  static __device__ __forceinline__ void pair(uint32_t w, float *a, float *b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    *a = f.x;
    *b = f.y;
  }
  static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) {
    const __half2 y = __hmax2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&y);
  }
};
template <> struct ScoreElem<float> {
  static __device__ __forceinline__ float one(float x) { return x; }
};

__device__ __forceinline__ void score_load32(const void *p, uint32_t *w) {
  asm("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}

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

template <typename E>
__device__ __forceinline__ float score_group(const uint32_t *w, float scale, ScoreSum &a) {
  float gm;
  if constexpr (sizeof(E) == 4) {
    gm = __uint_as_float(w[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) gm = fmaxf(gm, __uint_as_float(w[i]));
  } else {
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ScoreElem<E>::max(w[i], w[i + 8]);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < o; ++i) x[i] = ScoreElem<E>::max(x[i], x[i + o]);
    float u, v;
    ScoreElem<E>::pair(x[0], &u, &v);
    gm = fmaxf(u, v);
  }
  if (gm > a.m) a.raise(gm, scale);
  const float ref = a.m > -INFINITY ? a.m : 0.f;
  float2 s2 = make_float2(a.s, 0.f), t2 = make_float2(a.t, 0.f);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float2 x;
    if constexpr (sizeof(E) == 4) {
      if (i & 1) continue;
      x = make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1]));
    } else {
      ScoreElem<E>::pair(w[i], &x.x, &x.y);
    }
    score_pair(x, scale, ref, s2, t2);
  }
  a.s = s2.x + s2.y;
  a.t = t2.x + t2.y;
  return gm;
}

// A cluster of CTAs per row.  Groups of 64 bytes on 32-byte boundaries, a lane each; what a row has before its first boundary is
// group 0, what is behind the last whole group the last one (their elements one per lane, by the first warp of the row).
template <typename E>
__global__ void __launch_bounds__(SCORE_THREADS, 4) sx_score_kernel(const SxScoreArgs p, const E *__restrict__ logits, int64_t stride, int cluster) {
  constexpr int GE = SCORE_GROUP_BYTES / (int)sizeof(E);
  __shared__ ScoreShared sh;
  sx_pdl_wait();
  const int row = blockIdx.x / cluster, rank = blockIdx.x - row * cluster;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const E *x = logits + (int64_t)row * stride;
  const int lead = min(p.V, (int)((32u - ((uint32_t)(uintptr_t)x & 31u)) & 31u) / (int)sizeof(E));
  const int whole = (p.V - lead) / GE, rest = p.V - lead - whole * GE;
  const E *body = x + lead;
  ScoreSum a;
  ScoreList l;
  a.clear();
  l.clear();
  const int at = rank * SCORE_WARPS + warp, all = cluster * SCORE_WARPS;
  const auto edge = [&](const E *from, int n, int id) {
    const float v = lane < n ? ScoreElem<E>::one(from[lane]) : -INFINITY;
    if (v > a.m) a.raise(v, p.scale);
    float2 s2 = make_float2(a.s, 0.f), t2 = make_float2(a.t, 0.f);
    score_pair(make_float2(v, -INFINITY), p.scale, a.m > -INFINITY ? a.m : 0.f, s2, t2);
    a.s = s2.x;
    a.t = t2.x;
    const float gm = sx_warp_max(v);
    if (p.top) l.offer(gm, id, lane == 0 && gm > -INFINITY, p.top, lane);
  };
  if (at == 0 && lead) edge(x, lead, 0);
  uint32_t w[16];
  int g = at * 32 + lane;
  if (g < whole) { score_load32(body + (int64_t)g * GE, w); score_load32(body + (int64_t)g * GE + GE / 2, w + 8); }
#pragma unroll 1
  for (; g - lane < whole; g += all * 32) {
    uint32_t n[16];
    const int next = g + all * 32;
    if (next < whole) { score_load32(body + (int64_t)next * GE, n); score_load32(body + (int64_t)next * GE + GE / 2, n + 8); }
    float gm = -INFINITY;
    if (g < whole) gm = score_group<E>(w, p.scale, a);
    if (p.top) l.offer(gm, g + 1, g < whole && gm > -INFINITY, p.top, lane);
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = n[i];
  }
  if (at == 0 && rest) edge(body + (int64_t)whole * GE, rest, whole + 1);
  score_block_sum(sh, a, p.scale);
  if (p.top) {
    score_best_groups(sh, l, p.top);
    const float kth = sh.group[p.top - 1] ? sx_pack_value(sh.group[p.top - 1]) : -INFINITY;
    for (int i = warp; i < p.top; i += SCORE_WARPS) {
      if (!sh.group[i]) break;
      const int id = (int)sx_pack_index(sh.group[i]);
      const int from = id == 0 ? 0 : lead + (id - 1) * GE, n = id == 0 ? lead : id == whole + 1 ? rest : GE;
      if (lane < n) score_candidate(sh, ScoreElem<E>::one(x[from + lane]), from + lane, kth);
    }
    __syncthreads();
    score_rank(sh.cand, sh.n_cand, p.top, sh.best);
    __syncthreads();
  }
  const unsigned long long *best = sh.best;
  if (cluster > 1) {
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    if (rank == 0) {
      // the other CTAs' sums and lists; the lists side by side, then ranked together
      if (warp == 0) {
        ScoreSum b;
        b.clear();
        if (lane < cluster) {
          const ScoreShared *o = cl.map_shared_rank(&sh, lane);
          b.m = o->row[0]; b.s = o->row[1]; b.t = o->row[2];
        }
        b.warp_join(p.scale);
        __syncwarp();
        if (lane == 0) { sh.row[0] = b.m; sh.row[1] = b.s; sh.row[2] = b.t; }
      }
      for (int i = threadIdx.x; i < cluster * p.top; i += SCORE_THREADS)
        sh.cand[i] = cl.map_shared_rank(&sh, i / p.top)->best[i % p.top];
      __syncthreads();
      if (p.top) score_rank(sh.cand, cluster * p.top, p.top, sh.list);
      __syncthreads();
      best = sh.list;
    }
    cl.sync();                                   // no CTA leaves while its shared memory is read
    if (rank != 0) return;
  }
  score_write(sh, p, row, best, [&](int i) { return ScoreElem<E>::one(x[i]); });
}

// ---- entry point -----------------------------------------------------------------------------------------------------------
static bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }
static bool aligned4(const void *p) { return ((uintptr_t)p & 3) == 0; }

static sx_status score_args(int32_t T, int32_t V, int32_t n_given, const int32_t *tok_d, float temperature, int32_t top,
                            const sx_logprob_out *out, int32_t *status_d, SxScoreArgs *p) {
  if (!out || !status_d || T < 0 || V < 1 || n_given < 0 || top < 0) return SX_ERR_INVALID_ARG;
  if (n_given > SX_MAX_GIVEN || top > SX_MAX_ALTERNATIVES || V > SX_MAX_SCORE_VOCAB) return SX_ERR_UNSUPPORTED;
  if (!(temperature > 0.f && temperature < INFINITY) || !(1.0 / (double)temperature < 1e30)) return SX_ERR_INVALID_ARG;
  if (n_given > 0 && (!tok_d || !out->logp_d)) return SX_ERR_INVALID_ARG;
  if (top > 0 && !out->top_tok_d && !out->top_logp_d) return SX_ERR_INVALID_ARG;
  if (!aligned4(tok_d) || !aligned4(out->logp_d) || !aligned4(out->entropy_d) || !aligned4(out->top_tok_d) || !aligned4(out->top_logp_d))
    return SX_ERR_INVALID_ARG;
  memset(p, 0, sizeof(*p));
  p->T = T; p->V = V; p->n_given = n_given; p->top = top;
  p->scale = (float)(1.4426950408889634074 / (double)temperature);
  p->inverse = (float)(1.0 / (double)temperature);
  p->tok = tok_d;
  p->logp = out->logp_d; p->entropy = out->entropy_d; p->top_tok = out->top_tok_d; p->top_logp = out->top_logp_d;
  p->status = status_d;
  return SX_OK;
}

static int sms_of_current_device() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return n;
}

extern "C" sx_status sx_logprobs(int32_t dtype, int32_t T, int32_t V, const void *logits_d, int64_t stride, int32_t n_given,
                                 const int32_t *tok_d, float temperature, int32_t top, const sx_logprob_out *out, int32_t *status_d,
                                 void *stream) {
  SxScoreArgs p;
  SX_TRY(score_args(T, V, n_given, tok_d, temperature, top, out, status_d, &p));
  if (dtype < SX_BF16 || dtype > SX_F32 || !aligned16(logits_d) || stride < V) return SX_ERR_INVALID_ARG;
  if (T == 0) return SX_OK;
  const int sm = sms_of_current_device();
  if (!sm) return SX_ERR_CUDA;
  // CTAs per row: until there are four per SM, as long as each has two groups per lane
  const int64_t groups = (int64_t)V * (dtype == SX_F32 ? 4 : 2) / SCORE_GROUP_BYTES;
  int cluster = 1;
  while (cluster < SCORE_MAX_CLUSTER && (int64_t)T * cluster < 4 * sm && groups >= (int64_t)cluster * 2 * SCORE_THREADS) cluster *= 2;
  if ((int64_t)T * cluster > 0x7fffffffll) return SX_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(T * cluster)), block(SCORE_THREADS);
  cudaStream_t st = (cudaStream_t)stream;
  switch (dtype) {
    case SX_BF16: return sx_rc(sx_launch_cluster(sx_score_kernel<bf16>, grid, block, 0, (unsigned)cluster, st, p, (const bf16 *)logits_d, stride, cluster));
    case SX_F16: return sx_rc(sx_launch_cluster(sx_score_kernel<__half>, grid, block, 0, (unsigned)cluster, st, p, (const __half *)logits_d, stride, cluster));
    default: return sx_rc(sx_launch_cluster(sx_score_kernel<float>, grid, block, 0, (unsigned)cluster, st, p, (const float *)logits_d, stride, cluster));
  }
}
