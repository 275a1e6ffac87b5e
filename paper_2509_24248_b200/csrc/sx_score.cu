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
// others are before it, and the elements of the k best groups go through lists of the same kind.  The cost does not depend on
// the values but for the number of insertions.
//
// Measured: 4096 rows of 151936 in bf16 with five alternatives 217-256 us on different boxes (1.24 GB, 4.9-5.7 TB/s; 190 us at the copy
// rate), one row with twenty 12.7-13.9 us, 244 rows of 32001 in fp32, half of them masked, 15.2 us.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "sx_kernels.cuh"
#include "sx_launch.cuh"
#include "sx_score.cuh"

namespace cg = cooperative_groups;

#define SCORE_GROUP_BYTES 64
#define SCORE_MAX_WARPS 8              // warps of a CTA, which has one row
#define SCORE_MAX_CLUSTER 8            // CTAs of a row
static_assert(SX_MAX_GIVEN <= 64 && SX_MAX_ALTERNATIVES <= 32, "two given tokens per lane of the smallest CTA, a lane per alternative");

struct SxScoreArgs {
  int T, V, n_given, top;
  float scale, inverse;                // log2(e) / temperature, 1 / temperature
  const int32_t *tok;
  float *logp, *entropy, *top_logp;
  int32_t *top_tok, *status;
};

// The 32 best entries that a warp has met, as packed (value, id) keys: best first, lane by lane; 0 = none.
struct ScoreList {
  unsigned long long key;
  float floor;                         // value of the top-th entry, -inf while there is none
  __device__ __forceinline__ void clear() { key = 0ull; floor = -INFINITY; }
  static __device__ __forceinline__ unsigned long long step(unsigned long long k, int stride, bool larger) {
    const unsigned long long o = __shfl_xor_sync(0xffffffffu, k, stride);
    return (o > k) == larger ? o : k;
  }
  // the keys k of the lanes in m
  __device__ __forceinline__ void take(unsigned long long k, uint32_t m, int top, int lane) {
    if (__popc(m) > 8) {
      // sort the new ones (a bitonic network over the lanes, descending), then the better half of both lists, which is bitonic
      unsigned long long n = m >> lane & 1 ? k : 0ull;
#pragma unroll
      for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int stride = size / 2; stride > 0; stride /= 2) n = step(n, stride, ((lane & size) == 0) == ((lane & stride) == 0));
      n = __shfl_sync(0xffffffffu, n, 31 - lane);
      key = n > key ? n : key;
#pragma unroll
      for (int stride = 16; stride > 0; stride /= 2) key = step(key, stride, (lane & stride) == 0);
    } else {
      while (m) {
        const unsigned long long n = __shfl_sync(0xffffffffu, k, __ffs(m) - 1);
        m &= m - 1;
        const int at = __popc(__ballot_sync(0xffffffffu, key > n));
        const unsigned long long up = __shfl_up_sync(0xffffffffu, key, 1);
        if (lane > at) key = up;
        if (lane == at) key = n;
      }
    }
    const unsigned long long kth = __shfl_sync(0xffffffffu, key, top - 1);
    floor = kth ? sx_pack_value(kth) : -INFINITY;
  }
  // Groups: ids ascend with the lanes and from call to call, so one that only equals the floor is not among the first `top`.
  // shared: the floor of some warp of the CTA, the largest but for races.  A group below any warp's floor is not among the best of
  // the row, so whatever is read here lets enough through and the result does not depend on it.
  __device__ __forceinline__ void offer_group(float v, int id, int top, int lane, volatile float *shared) {
    const bool on = v > floor && v >= *shared;
    const uint32_t m = __ballot_sync(0xffffffffu, on);
    if (m == 0) return;
    take(sx_pack(v + 0.f, (uint32_t)id), m, top, lane);                  // -0 counts as 0
    if (lane == 0 && floor > *shared) *shared = floor;
  }
  // Entries in any order of ids; nothing below `least` is wanted.
  __device__ __forceinline__ void offer(float v, int id, float least, int top, int lane) {
    const unsigned long long k = v >= least && v > -INFINITY ? sx_pack(v + 0.f, (uint32_t)id) : 0ull;      // a NaN is not
    const unsigned long long kth = __shfl_sync(0xffffffffu, key, top - 1);
    const uint32_t m = __ballot_sync(0xffffffffu, k > kth);
    if (m) take(k, m, top, lane);
  }
};

struct ScoreShared {
  unsigned long long list[SCORE_MAX_WARPS * 32];                      // the lists of the warps, or of the CTAs of a cluster
  unsigned long long group[32], best[32];                             // the best groups, the best elements
  float sum[SCORE_MAX_WARPS][3], row[3];
  volatile float floor;
};
static_assert(SCORE_MAX_CLUSTER <= SCORE_MAX_WARPS, "the lists of a cluster lie where those of the warps did");

// ---- steps shared by both forms; all W warps of the CTA call them ---------------------------------------------------
template <int W> __device__ __forceinline__ void score_sync() { if (W == 1) __syncwarp(); else __syncthreads(); }

// sums of the warps -> sh.row
template <int W>
__device__ __forceinline__ void score_join_sums(ScoreShared &sh, ScoreSum a, float scale) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  a.warp_join(scale);
  if (W > 1) {
    if (lane == 0) { sh.sum[warp][0] = a.m; sh.sum[warp][1] = a.s; sh.sum[warp][2] = a.t; }
    __syncthreads();
    if (warp == 0) {
      a.clear();
      if (lane < W) { a.m = sh.sum[lane][0]; a.s = sh.sum[lane][1]; a.t = sh.sum[lane][2]; }
      a.warp_join(scale);
    }
  }
  if (threadIdx.x == 0) { sh.row[0] = a.m; sh.row[1] = a.s; sh.row[2] = a.t; }
  score_sync<W>();
}

// The `top` best of n descending lists of 32 in sh.list -> dst, best first, 0 behind the last: an entry's place is the number of
// entries before it, found in every list by halving.
template <int W>
__device__ __forceinline__ void score_join_lists(ScoreShared &sh, int n, int top, unsigned long long *dst) {
  if (threadIdx.x < 32) dst[threadIdx.x] = 0ull;
  score_sync<W>();
  for (int e = threadIdx.x; e < n * top; e += W * 32) {
    const unsigned long long mine = sh.list[e / top * 32 + e % top];
    int rank = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const unsigned long long *p = sh.list + i * 32;
      int lo = 0;
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
        if (p[lo + step - 1] > mine) lo += step;
      rank += lo + (p[lo] > mine ? 1 : 0);
    }
    if (mine && rank < top) dst[rank] = mine;
  }
  score_sync<W>();
}
template <int W>
__device__ __forceinline__ void score_join_warps(ScoreShared &sh, const ScoreList &l, int top, unsigned long long *dst) {
  if (W == 1) {
    dst[threadIdx.x] = (int)threadIdx.x < top ? l.key : 0ull;
    __syncwarp();
  } else {
    sh.list[threadIdx.x] = l.key;
    score_join_lists<W>(sh, W, top, dst);
  }
}

// The sums and the lists of groups of a row's CTAs -> sh.row, sh.group of the first of them; false in the others, which are done.
template <int W>
__device__ __forceinline__ bool score_join_cluster(ScoreShared &sh, int cluster, int rank, int top, float scale) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  cg::cluster_group cl = cg::this_cluster();
  cl.sync();
  if (rank == 0) {
    if (warp == 0) {
      ScoreSum b;
      b.clear();
      if (lane < cluster) {
        const ScoreShared *o = cl.map_shared_rank(&sh, lane);
        b.m = o->row[0]; b.s = o->row[1]; b.t = o->row[2];
      }
      b.warp_join(scale);
      if (lane == 0) { sh.row[0] = b.m; sh.row[1] = b.s; sh.row[2] = b.t; }
    }
    if (top)
      for (int i = threadIdx.x; i < cluster * 32; i += W * 32) sh.list[i] = cl.map_shared_rank(&sh, i / 32)->group[i % 32];
  }
  cl.sync();                                   // no CTA leaves while its shared memory is read
  if (rank != 0) return false;
  if (top) score_join_lists<W>(sh, cluster, top, sh.group);
  return true;
}

// The best elements of the best groups -> sh.best.  element(group id, lane, &index): the lane's element, -inf: none.  What is below the
// maximum of the last of the groups is below `top` others.
template <int W, typename F>
__device__ __forceinline__ void score_best_elements(ScoreShared &sh, int top, F element) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float least = sh.group[top - 1] ? sx_pack_value(sh.group[top - 1]) : -INFINITY;
  ScoreList l;
  l.clear();
  // four groups' elements on the way at a time
#pragma unroll 1
  for (int i = warp; i < top; i += 4 * W) {
    float v[4];
    int index[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned long long g = i + j * W < top ? sh.group[i + j * W] : 0ull;
      v[j] = -INFINITY;
      index[j] = 0;
      if (g != 0ull) v[j] = element((int)sx_pack_index(g), lane, &index[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) l.offer(v[j], index[j], least, top, lane);
  }
  score_join_warps<W>(sh, l, top, sh.best);
}

// The given tokens of a row and their logits, which are on their way during the pass.
template <int W> struct ScoreGiven {
  enum { N = W == 1 ? 2 : 1 };
  int tok[N];
  float x[N];
  template <typename F>
  __device__ __forceinline__ void fetch(const SxScoreArgs &p, int row, F logit) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = threadIdx.x + j * W * 32;
      tok[j] = -1;
      x[j] = 0.f;
      if (i < p.n_given) {
        tok[j] = p.tok[(int64_t)row * p.n_given + i];
        if (tok[j] >= 0 && tok[j] < p.V) x[j] = logit(tok[j]);
      }
    }
  }
};

// Results of a row.  A row with a NaN or an infinite logit has no probabilities: NaN, and no alternatives; where every logit is -inf
// no token has any.
template <int W>
__device__ __forceinline__ void score_write(const ScoreShared &sh, const SxScoreArgs &p, int row, const ScoreGiven<W> &given) {
  const float m = sh.row[0], s = sh.row[1], t = sh.row[2], LN2 = 0.6931471805599453f, NaN = __int_as_float(0x7fffffff);
  const bool bad = !(s >= 0.f) || m == INFINITY, none = !bad && m == -INFINITY;
  const float ln = none ? 0.f : logf(s);
  const auto log_p = [&](float x) { return fmaf(fmaf(x, 0.5f, -0.5f * m), 2.f * p.inverse, -ln); };      // as score_gap
#pragma unroll
  for (int j = 0; j < ScoreGiven<W>::N; ++j) {
    const int i = threadIdx.x + j * W * 32;
    if (i < p.n_given) {
      float y = 0.f;
      if (given.tok[j] >= 0 && given.tok[j] < p.V) {
        y = bad ? NaN : given.x[j] == -INFINITY ? -INFINITY : log_p(given.x[j]);
      } else if (given.tok[j] != -1) {
        y = NaN;
        sx_set_status(p.status, SX_ERR_CAPACITY);
      }
      p.logp[(int64_t)row * p.n_given + i] = y;
    }
  }
  if (p.entropy && threadIdx.x == 0) p.entropy[row] = bad ? NaN : none ? 0.f : ln - LN2 * (t / s);
  if ((int)threadIdx.x < p.top) {
    const unsigned long long key = sh.best[threadIdx.x];
    const int64_t at = (int64_t)row * p.top + threadIdx.x;
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

// Volatile, with a clobber and on the coherent path: the kernel may start while the one that writes the logits still runs, so no load of
// them may move before sx_pdl_wait (nor is `logits` __restrict__, which would allow the non-coherent path for the others).
__device__ __forceinline__ void score_load32(const void *p, uint32_t *w) {
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}

template <typename E>
__device__ __forceinline__ float score_group_max(const uint32_t *w) {
  if constexpr (sizeof(E) == 4) {
    float gm = __uint_as_float(w[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) gm = fmaxf(gm, __uint_as_float(w[i]));
    return gm;
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
    return fmaxf(u, v);
  }
}
// f(pair of neighbouring elements) for all of a group
template <typename E, typename F>
__device__ __forceinline__ void score_pairs(const uint32_t *w, F f) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float2 x;
    if constexpr (sizeof(E) == 4) {
      if (i & 1) continue;
      x = make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1]));
    } else {
      ScoreElem<E>::pair(w[i], &x.x, &x.y);
    }
    f(x);
  }
}

// The sums of a lane over its groups.  Issue slots bound this pass, so the plain way takes as few as it can: d = fma(x, c, -r),
// r = fl(c m), with sums relative to 2^r, and a new reference only where a group is more than 2^SCORE_SLACK above the old one.
// It has no place for logits so large that the rounding of r counts (a type's lowest value among them, where a row has nothing
// else): the first such group turns the warp over to the careful way for the rest of the row (score_pair: one more
// instruction an element), whose sums are relative to 2^(c m).  r is off by fma(m, c, -r), exactly; the two differ by that power
// of two.
#define SCORE_SLACK 4.f
struct ScorePlain {
  ScoreSum a;
  float r, limit;                  // limit: a group maximum above it asks for a new reference
  __device__ __forceinline__ void clear() { a.clear(); r = 0.f; limit = -INFINITY; }
  // false: not added, the careful way has to
  template <typename E>
  __device__ __forceinline__ bool add(const uint32_t *w, float gm, bool on, float scale, float slack) {
    if (on && gm > limit) {
      const float to = gm * scale;
      if (a.m > -INFINITY) {
        const float d = fmaxf(r - to, -200.f), f = score_exp2(d);
        a.t = f * fmaf(a.s, d, a.t);
        a.s *= f;
      }
      a.m = gm;
      r = to;
      limit = fminf(gm + slack, 3.402823466e38f);     // an infinite logit is above it at any temperature
    }
    float s0 = 0.f, s1 = 0.f, t0 = 0.f, t1 = 0.f;       // of this group: short sums of small numbers, added to the long ones once
    score_pairs<E>(w, [&](float2 x) {
      const float d0 = score_max_nan(fmaf(x.x, scale, -r), -200.f), d1 = score_max_nan(fmaf(x.y, scale, -r), -200.f);
      const float e0 = score_exp2(d0), e1 = score_exp2(d1);
      s0 += e0;
      s1 += e1;
      t0 = fmaf(e0, d0, t0);
      t1 = fmaf(e1, d1, t1);
    });
    if (!__all_sync(0xffffffffu, !on || fabsf(r) < 1048576.f)) return false;
    if (on) { a.s += s0 + s1; a.t += t0 + t1; }
    return true;
  }
  // relative to 2^(c m) from here on
  __device__ __forceinline__ ScoreSum exact(float scale) {
    if (a.s != 0.f) {
      const float off = fmaf(a.m, scale, -r), f = score_exp2(-off);
      a.t = f * fmaf(-off, a.s, a.t);
      a.s *= f;
    }
    return a;
  }
};

// W warps per CTA, a cluster of CTAs per row.  Groups of 64 bytes on 32-byte boundaries, a lane each; what a row has before its
// first boundary is group 0, what is behind the last whole group the last one (their elements one per lane, by the first
// warp of the row).
template <typename E, int W>
__global__ void __launch_bounds__(W * 32, 32 / W) sx_score_kernel(const SxScoreArgs p, const E *logits, int64_t stride, int cluster) {
  constexpr int GE = SCORE_GROUP_BYTES / (int)sizeof(E);
  __shared__ ScoreShared sh;
  if (threadIdx.x == 0) sh.floor = -INFINITY;
  score_sync<W>();
  sx_pdl_wait();
  const int row = blockIdx.x / cluster, rank = blockIdx.x - row * cluster;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const E *x = logits + (int64_t)row * stride;
  const int lead = min(p.V, (int)((32u - ((uint32_t)(uintptr_t)x & 31u)) & 31u) / (int)sizeof(E));
  const int whole = (p.V - lead) / GE, rest = p.V - lead - whole * GE;
  const E *body = x + lead;
  ScoreGiven<W> given;
  if (rank == 0) given.fetch(p, row, [&](int i) { return ScoreElem<E>::one(x[i]); });
  ScoreList l;
  l.clear();
  const int at = rank * W + warp, stride_g = cluster * W * 32;
  // the elements before and behind the groups, one per lane; their sums are added last
  const float e0 = at == 0 && lane < lead ? ScoreElem<E>::one(x[lane]) : -INFINITY;
  const float e1 = at == 0 && lane < rest ? ScoreElem<E>::one(body[(int64_t)whole * GE + lane]) : -INFINITY;
  if (p.top && at == 0 && lead) {
    const float gm = sx_warp_max(e0);
    l.offer_group(lane == 0 ? gm : -INFINITY, 0, p.top, lane, &sh.floor);
  }
  // a lane without a group reads the last one again (a load under a condition costs a move for every word)
  const auto load = [&](int g, uint32_t *w) {
    const E *from = body + (int64_t)min(g, whole - 1) * GE;
    score_load32(from, w);
    score_load32(from + GE / 2, w + 8);
  };
  int g = at * 32 + lane;
  ScoreSum a;
  {
    ScorePlain f;
    f.clear();
    const float slack = SCORE_SLACK / p.scale;
    uint32_t w0[16], w1[16];
    const auto take = [&](const uint32_t *w) {
      const bool on = g < whole;
      const float gm = on ? score_group_max<E>(w) : -INFINITY;
      if (!f.add<E>(w, gm, on, p.scale, slack)) return false;
      if (p.top) l.offer_group(gm, g + 1, p.top, lane, &sh.floor);
      g += stride_g;
      return true;
    };
    if (g - lane < whole) load(g, w0);
#pragma unroll 1
    while (g - lane < whole) {
      load(g + stride_g, w1);
      if (!take(w0)) break;
      if (g - lane >= whole) break;
      load(g + stride_g, w0);
      if (!take(w1)) break;
    }
    a = f.exact(p.scale);
  }
#pragma unroll 1
  for (; g - lane < whole; g += stride_g) {     // the careful way
    uint32_t w[16];
    load(g, w);
    const float gm = g < whole ? score_group_max<E>(w) : -INFINITY;
    if (g < whole) {
      if (gm > a.m) a.raise(gm, p.scale);
      const float ref = a.m > -INFINITY ? a.m : 0.f;
      float2 s2 = make_float2(0.f, 0.f), t2 = s2;
      score_pairs<E>(w, [&](float2 v) { score_pair(v, p.scale, ref, s2, t2); });
      a.s += s2.x + s2.y;
      a.t += t2.x + t2.y;
    }
    if (p.top) l.offer_group(gm, g + 1, p.top, lane, &sh.floor);
  }
  if (at == 0 && lead + rest) {
    const float gm = sx_warp_max(e1);
    if (p.top && rest) l.offer_group(lane == 0 ? gm : -INFINITY, whole + 1, p.top, lane, &sh.floor);
    const float top = fmaxf(e0, e1);
    if (top > a.m) a.raise(top, p.scale);
    float2 s2 = make_float2(a.s, 0.f), t2 = make_float2(a.t, 0.f);
    score_pair(make_float2(e0, e1), p.scale, a.m > -INFINITY ? a.m : 0.f, s2, t2);
    a.s = s2.x + s2.y;
    a.t = t2.x + t2.y;
  }
  score_join_sums<W>(sh, a, p.scale);
  if (p.top) score_join_warps<W>(sh, l, p.top, sh.group);
  if constexpr (W == SCORE_MAX_WARPS) {
    if (cluster > 1 && !score_join_cluster<W>(sh, cluster, rank, p.top, p.scale)) return;
  }
  if (p.top)
    score_best_elements<W>(sh, p.top, [&](int id, int i, int *index) {
      const int from = id == 0 ? 0 : lead + (id - 1) * GE, n = id == 0 ? lead : id == whole + 1 ? rest : GE;
      *index = from + i;
      return i < n ? ScoreElem<E>::one(x[from + i]) : -INFINITY;
    });
  score_write<W>(sh, p, row, given);
}

// ---- from hidden states: what the product left ---------------------------------------------------------------------------
// A cluster of CTAs per row: sums of the parts of the vocabulary, maxima of groups of 32 logits, and the logits (all laid out for the
// threads that write them, see SxScoreOut; -inf behind the vocabulary).
__global__ void __launch_bounds__(SCORE_MAX_WARPS * 32) sx_score_head_kernel(const SxScoreArgs p, const SxScoreOut o, int row0, int parts, int tiles, int cluster) {
  constexpr int W = SCORE_MAX_WARPS;
  __shared__ ScoreShared sh;
  if (threadIdx.x == 0) sh.floor = -INFINITY;
  __syncthreads();
  sx_pdl_launch_dependents();
  sx_pdl_wait();
  const int row = blockIdx.x / cluster, rank = blockIdx.x - row * cluster, lane = threadIdx.x & 31, groups = tiles * 4;
  const int first = rank * W * 32 + threadIdx.x, step = cluster * W * 32;
  ScoreGiven<W> given;
  if (rank == 0) given.fetch(p, row0 + row, [&](int i) { return o.logits[sx_score_at(o, row, i)]; });
  const auto maximum = [&](int g) { return g < groups ? o.maxima[((size_t)(g >> 2) * o.rows + row) * 4 + (g & 3)] : -INFINITY; };
  float ahead[4];                               // the first maxima are on their way while the sums are joined
#pragma unroll
  for (int j = 0; j < 4; ++j) ahead[j] = p.top ? maximum(first + j * step) : -INFINITY;
  ScoreSum a;
  a.clear();
#pragma unroll 4
  for (int i = first; i < parts; i += step) {
    const float *from = o.sums + ((size_t)i * o.rows + row) * 3;
    a.join(from[0], from[1], from[2], p.scale);
  }
  score_join_sums<W>(sh, a, p.scale);
  if (p.top) {
    ScoreList l;
    l.clear();
    for (int g = first; g - lane < groups; g += 4 * step) {
      float v[4];
      int best = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = ahead[j];
        ahead[j] = maximum(g + (4 + j) * step);
        if (v[j] > v[best]) best = j;
      }
      // the best of a lane's four first: hardly any of the others is above what the list then begins with
      const float b = v[best];
      l.offer(b, g + best * step, sh.floor, p.top, lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) l.offer(j == best ? -INFINITY : v[j], g + j * step, sh.floor, p.top, lane);
      if (lane == 0 && l.floor > sh.floor) sh.floor = l.floor;
    }
    score_join_warps<W>(sh, l, p.top, sh.group);
  }
  if (cluster > 1 && !score_join_cluster<W>(sh, cluster, rank, p.top, p.scale)) return;
  if (p.top)
    score_best_elements<W>(sh, p.top, [&](int id, int i, int *index) {
      *index = id * 32 + i;
      return o.logits[sx_score_at(o, row, id * 32 + i)];
    });
  score_write<W>(sh, p, row0 + row, given);
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

// Warps and CTAs per row.  An SM has room for 32 warps of this kernel.  A row's ends (first loads, joining, alternatives: 3 to 5 us in
// which it reads nothing) are shorter the fewer warps it has, and weigh less the longer it takes; so a row has as many warps as
// there is room for with all rows at once (4096 rows of 32000 in bf16 with 1, 2, 4, 8: 61, 69, 76, 92 us; 2000 of 50000: 56, 52, 56,
// 63; 1000 of 32000: 29, 25, 24, 27; 1500 of 151936: 123, 104, 100, 98; 4096 of them 219, 219, 217, 237), and every warp two rounds of
// groups, where the row has as many.  A row is spread over a cluster while that makes no more than 1.75 CTAs per SM and leaves
// each warp a round (one row of 151936 in bf16 on 1, 2, 4, 8 CTAs: 22, 19, 15.6, 13.9 us; 74 rows: 19.3, 16.4, 17.6, 22 us).
struct ScoreSplit { int warps, cluster; };
static ScoreSplit score_split(int64_t T, int64_t groups, int sm) {
  const int64_t room = 32ll * sm, most = groups / (2 * 32);
  ScoreSplit n = {1, 1};
  while (n.warps < SCORE_MAX_WARPS && n.warps * 2 <= most && T * n.warps * 2 <= room) n.warps *= 2;
  while (n.cluster < SCORE_MAX_CLUSTER && n.warps == SCORE_MAX_WARPS && groups >= 32ll * n.warps * n.cluster * 2 && 4 * T * n.cluster * 2 <= 7ll * sm)
    n.cluster *= 2;
  return n;
}

template <typename E, int W>
static sx_status launch_score_of(const SxScoreArgs &p, const E *x, int64_t stride, int cluster, cudaStream_t st) {
  // (a cluster of one is not launched as one: that leaves room for fewer CTAs, 4096 rows of 515 in 30 instead of 12 us)
  const dim3 grid((unsigned)(p.T * cluster)), block(W * 32);
  if constexpr (W == SCORE_MAX_WARPS) {
    if (cluster > 1) return sx_rc(sx_launch_cluster(sx_score_kernel<E, W>, grid, block, 0, (unsigned)cluster, st, p, x, stride, cluster));
  }
  return sx_rc(sx_launch(sx_score_kernel<E, W>, grid, block, 0, st, p, x, stride, 1));
}
template <typename E>
static sx_status launch_score(const SxScoreArgs &p, const void *logits, int64_t stride, ScoreSplit n, cudaStream_t st) {
  const E *x = (const E *)logits;
  switch (n.warps) {
    case 1: return launch_score_of<E, 1>(p, x, stride, n.cluster, st);
    case 2: return launch_score_of<E, 2>(p, x, stride, n.cluster, st);
    case 4: return launch_score_of<E, 4>(p, x, stride, n.cluster, st);
    default: return launch_score_of<E, 8>(p, x, stride, n.cluster, st);
  }
}

extern "C" sx_status sx_logprobs(int32_t dtype, int32_t T, int32_t V, const void *logits_d, int64_t stride, int32_t n_given,
                                 const int32_t *tok_d, float temperature, int32_t top, const sx_logprob_out *out, int32_t *status_d,
                                 void *stream) {
  SxScoreArgs p;
  SX_TRY(score_args(T, V, n_given, tok_d, temperature, top, out, status_d, &p));
  if (dtype < SX_BF16 || dtype > SX_F32 || !logits_d || (uintptr_t)logits_d % (dtype == SX_F32 ? 4 : 2) || stride < V) return SX_ERR_INVALID_ARG;
  if (T == 0) return SX_OK;
  const int sm = sx_sm_count();
  if (!sm) return SX_ERR_CUDA;
  const int64_t groups = (int64_t)V * (dtype == SX_F32 ? 4 : 2) / SCORE_GROUP_BYTES;
  const ScoreSplit n = score_split(T, groups, sm);
  if ((int64_t)T * n.cluster > 0x7fffffffll) return SX_ERR_UNSUPPORTED;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == SX_BF16) return launch_score<bf16>(p, logits_d, stride, n, st);
  if (dtype == SX_F16) return launch_score<__half>(p, logits_d, stride, n, st);
  return launch_score<float>(p, logits_d, stride, n, st);
}

// Rows are taken SX_SCORE_MAX_PART at a time at most, in as few equal parts as that allows: every part reads the whole head.
static int score_part(int T) {
  const int parts = 1 + (T - 1) / SX_SCORE_MAX_PART;        // rounded up; T may be as large as 32 bits hold
  return 1 + (T - 1) / parts;
}

struct ScoreWs { size_t logits, maxima, sums, total; };
static ScoreWs score_ws(int rows, int V, int sm) {
  const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const size_t tiles = (V + SX_TILE_M - 1) / SX_TILE_M, parts = rows > SX_SCORE_FEW || tiles < (size_t)sm ? tiles : (size_t)sm;
  ScoreWs w;
  w.logits = 0;
  w.maxima = up(rows * tiles * SX_TILE_M * sizeof(float));
  w.sums = w.maxima + up(rows * tiles * 4 * sizeof(float));
  w.total = w.sums + up(parts * rows * 3 * sizeof(float));
  return w;
}

extern "C" size_t sx_head_logprobs_ws_bytes(int32_t T, int32_t V) {
  const int sm = sx_sm_count();
  if (T < 1 || V < 1 || V > SX_MAX_SCORE_VOCAB || !sm) return 0;
  return score_ws(score_part(T), V, sm).total;
}

extern "C" sx_status sx_head_logprobs(const void *head_d, int32_t tiled, int32_t V, int32_t H, int32_t T, const void *hidden_d,
                                      int32_t n_given, const int32_t *tok_d, float temperature, int32_t top,
                                      const sx_logprob_out *out, void *ws_d, size_t ws_bytes, int32_t *status_d, void *stream) {
  SxScoreArgs p;
  SX_TRY(score_args(T, V, n_given, tok_d, temperature, top, out, status_d, &p));
  if (!aligned16(head_d) || !aligned16(hidden_d) || (tiled != 0 && tiled != 1)) return SX_ERR_INVALID_ARG;
  if (H < 8 || H % 8 || ((int64_t)V + 255) * (H + 63) / 64 > 0x7fffffff) return SX_ERR_UNSUPPORTED;     // boxes of a repacked head
  if (T == 0) return SX_OK;
  int dev = 0, sm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || !(sm = sx_sm_count())) return SX_ERR_CUDA;
  const int part = score_part(T);
  const ScoreWs w = score_ws(part, V, sm);
  if (!ws_d || ((uintptr_t)ws_d & 255) || ws_bytes < w.total) return SX_ERR_WORKSPACE;
  if (part <= SX_SCORE_FEW) SX_TRY(sx_gemm_init(dev));
  SxScoreOut o;
  o.scale = p.scale;
  o.logits = (float *)((char *)ws_d + w.logits);
  o.maxima = (float *)((char *)ws_d + w.maxima);
  o.sums = (float *)((char *)ws_d + w.sums);
  o.rows = part;
  const bf16 *head = (const bf16 *)head_d, *rows = (const bf16 *)hidden_d;
  const int tiles = (V + SX_TILE_M - 1) / SX_TILE_M;
  cudaStream_t st = (cudaStream_t)stream;
  for (int r0 = 0, R; r0 < T; r0 += R) {
    R = T - r0 < part ? T - r0 : part;
    int parts = 0;
    if (part <= SX_SCORE_FEW) SX_TRY(sx_launch_score_head(head, tiled != 0, V, H, rows + (size_t)r0 * H, R, o, &parts, sm, status_d, st));
    else SX_TRY(sx_launch_score_pairs(head, tiled != 0, V, H, rows + (size_t)r0 * H, R, o, &parts, status_d, st));
    // CTAs per row: as many as there is room for at a time, four rounds of groups for each.  (Twice as many end 3 us sooner by
    // themselves, but keep the next call's product off twice as many SMs: 7 rows 221 instead of 217 us in a row of calls.)
    int cluster = 1;
    while (cluster < SCORE_MAX_CLUSTER && R * cluster * 2 <= 4 * sm && tiles * 4 >= cluster * 2 * 4 * SCORE_MAX_WARPS * 32) cluster *= 2;
    const dim3 grid(R * cluster), block(SCORE_MAX_WARPS * 32);
    if (cluster > 1) SX_TRY(sx_rc(sx_launch_cluster(sx_score_head_kernel, grid, block, 0, (unsigned)cluster, st, p, o, r0, parts, tiles, cluster)));
    else SX_TRY(sx_rc(sx_launch(sx_score_head_kernel, grid, block, 0, st, p, o, r0, parts, tiles, 1)));
  }
  return SX_OK;
}
