// Shared pieces of the decode attention over the 8-bit paged cache (sx_attn8.cu, sx_attn8_tc.cu):
// parameters, the list of work and the addressing of partial results.
//
// Work.  A "unit" is a set of query rows that read the same slots: in the OWN list unit b is sequence b with its
// slots behind the shared prefix, in the PREFIX list unit g is a group of sequences with the prefix they share.  A
// unit has nq = rows * (query heads per KV head) queries per KV head, cut into tiles of at most `qt`; a list holds,
// in this order, the steps (runs of `step` slots) of every (unit, KV head, tile).  The list is cut into equal
// runs of `per` steps, whatever the lengths: run c (a warp or a CTA) takes steps [c * per, (c + 1) * per) and
// leaves one partial result for every (unit, head, tile) it meets.
//
// Partial results.  Row base of the partial of run c for (unit, head, tile): qt * c + cols(unit) + head * nq +
// tile * qt, where cols(unit) counts the queries of all units before it.  Going along the list either c grows by
// one (qt rows further) or the tile does (exactly its rows further), so no two partials overlap.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "sx_common.cuh"
#include "sx_launch.cuh"

#define A8_MAX_UNITS 1024          // sequences of one call (the plan of a list lives in shared memory)
#define A8_SPLIT_STEP 16           // slots per step of the warp-level kernel
#define A8_TC_STEP 128             // slots per step of the tensor-memory kernel
#define A8_MERGE_THREADS 256
// How far (in powers of two) a score may exceed its reference before the reference moves.  A weight then stays below
// 2^14 in fp16, whose subnormals reach down to 2^-24: whatever a row's largest weight is between 1 and 2^14, weights
// are held to 2^-25 of it or better.  One query that exceeds is enough to make a warp look at all of them.
#define A8_SLACK 14.f
// The tensor-memory kernel's partial outputs are in units of 2^A8_V_SHIFT (sx_attn8_tc.cu)
#define A8_V_SHIFT 44

struct SxA8List {                  // one list: what the main kernel writes down for the merge
  int32_t *cum;                    // [units] first list position of the unit (the host has checked that lists fit)
  int32_t *steps;                  // [units] steps of one (head, tile) of the unit
  int32_t *total;                  // [1]
  float2 *ml;                      // partial (reference, sum) per row
  float *o;                        // partial outputs [row][d]
  int qt, qt_shift, step, step_shift, runs, min_per, spread;
  int parts_shift;                 // log2 of the partial results per run and tile (the tensor-memory kernel's copies), `half`
  int64_t half;                    // rows apart
  float unit;                      // factor that brings this list's partial outputs to the merge's unit
};

struct SxA8 {
  int nq, nkv, G, d, page, B, rows, E, n_groups, max_pages, num_pages;
  float scale_log2;
  int64_t q_stride;                // elements between query rows
  const bf16 *q;
  const int32_t *cache_len, *page_table, *group_start, *prefix_len;
  const uint64_t *row_mask;        // [B * rows] or nullptr: every drafted slot
  const uint8_t *k, *v, *ks, *vs;
  bf16 *o_out;
  int32_t *status;
  int32_t *seq_group;              // [B] for the merge: group of a sequence, -1 when it shares nothing
  SxA8List own, pre;
  float unit;                      // the merge's unit: 2^A8_V_SHIFT where a list takes the tensor-memory kernel, else 1
  int early;                       // lengths and groups are inputs of the iteration: the plan may precede the wait
  int after_prefix;                // the own list's kernel: launched behind the prefix list's, see sx_attn8.cu
};

// Order of the launches.  The prefix list's kernel and the own list's do not depend on one another, so the second
// is not made to wait for the first: the prefix kernel lets its dependents start only after its own wait (all that came
// before has then completed), the own kernel starts without one and waits at its END - its completion then covers the
// prefix kernel's, as the merge kernel's wait needs it to.
template <bool PRE>
__device__ __forceinline__ void a8_enter(const SxA8 &p) {
  if (PRE) {
    if (!p.early) { sx_pdl_wait(); sx_pdl_launch_dependents(); }
  } else {
    sx_pdl_launch_dependents();
    if (!p.early && !p.after_prefix) sx_pdl_wait();
  }
}
template <bool PRE>
__device__ __forceinline__ void a8_planned(const SxA8 &p) {
  if (!p.early) return;
  if (PRE) { sx_pdl_wait(); sx_pdl_launch_dependents(); }
  else if (!p.after_prefix) sx_pdl_wait();
}
template <bool PRE>
__device__ __forceinline__ void a8_leave(const SxA8 &p) {
  if (!PRE && p.after_prefix) sx_pdl_wait();
}

// ---- the plan of a list in shared memory ------------------------------------------------------------------
struct A8Plan {
  int32_t *cum;                    // [units + 1]
  int32_t *steps;                  // [units] of one (head, tile)
  int32_t *len;                    // [B] cached slots (checked)
  int32_t *pre;                    // [B] slots that the shared prefix covers for the sequence
  int32_t *grp;                    // [B] group or -1
  int32_t *bad;                    // [n_groups]
  int units, per;
};
__host__ __device__ inline size_t a8_plan_bytes(int B, int n_groups) {
  return ((size_t)(B + 1) * 4 + (size_t)B * 16 + (size_t)(n_groups > 0 ? n_groups : 1) * 4 + 32 * 4 + 15) & ~(size_t)15;
}

// tiles of a unit with nq queries; steps of a run
__device__ __forceinline__ int a8_tiles(int nq, int qt_shift) { return (nq + (1 << qt_shift) - 1) >> qt_shift; }
// (at least min_per, what a run has in flight at once, as long as that leaves a run for every SM: three sequences of 129
// slots take 7.8 us with a step per run, 9.4 us with two and 11.9 us with four; one of 4096 slots 17.2 us with two, 15.2 us
// with four)
__device__ __forceinline__ int a8_per(int total, const SxA8List &ls) {
  const int least = min(ls.min_per, (int)((uint32_t)(total + ls.spread - 1) / (uint32_t)ls.spread));
  return max(max(least, 1), (int)((uint32_t)(total + ls.runs - 1) / (uint32_t)ls.runs));
}
// (align, the granule in which steps begin, is a power of two)
__device__ __forceinline__ int a8_first_slot(const A8Plan &pl, int b, int align) { return pl.pre[b] & ~(align - 1); }
__device__ __forceinline__ int a8_members(const SxA8 &p, int g) { return p.group_start[g + 1] - p.group_start[g]; }

// steps of one (head, tile) of unit u
template <bool PRE>
__device__ __forceinline__ int a8_steps(const SxA8 &p, const A8Plan &pl, const SxA8List &ls, int u, int align) {
  if (PRE) {
    const int b0 = p.group_start[u], b1 = p.group_start[u + 1];
    if (b1 <= b0 || pl.pre[b0] == 0) return 0;
    return (pl.pre[b0] + ls.step - 1) >> ls.step_shift;
  }
  const int cap = p.max_pages * p.page;
  const int end = min(pl.len[u] + p.E, cap), a0 = a8_first_slot(pl, u, align);
  // (a sequence without a slot behind the prefix has no steps: its table may have no page there)
  return end > pl.pre[u] ? (end - a0 + ls.step - 1) >> ls.step_shift : 0;
}
template <bool PRE>
__device__ __forceinline__ int a8_unit_nq(const SxA8 &p, int u) {
  return (PRE ? a8_members(p, u) : 1) * p.rows * p.G;
}

// Builds the plan with all threads of the CTA (NT of them).  Lengths and groups are checked on the way: what is out
// of range is reported and held to what exists; a group whose prefix is longer than a member's cache (or groups
// that do not cover the batch in order) is reported and its members read their own tables.
template <bool PRE, int NT>
__device__ void a8_plan(const SxA8 &p, const SxA8List &ls, int align, uint8_t *smem, A8Plan &pl) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pl.cum = reinterpret_cast<int32_t *>(smem);
  int32_t *wsum = pl.cum + p.B + 1;
  pl.steps = wsum + 32;
  pl.len = pl.steps + p.B;
  pl.pre = pl.len + p.B;
  pl.grp = pl.pre + p.B;
  pl.bad = pl.grp + p.B;
  pl.units = PRE ? p.n_groups : p.B;
  const int cap = p.max_pages * p.page;
  bool wrong = false;
  bool ordered = true;
#pragma unroll 1
  for (int g = tid; g < p.n_groups; g += NT) {
    pl.bad[g] = 0;
    const int s = p.group_start[g], e = p.group_start[g + 1];
    ordered = ordered && s >= 0 && s <= e && e <= p.B && (g > 0 || s == 0) && (g < p.n_groups - 1 || e == p.B);
  }
  ordered = __syncthreads_and(ordered) != 0;
#pragma unroll 1
  for (int b = tid; b < p.B; b += NT) {
    int n = p.cache_len[b];
    if (n < 0 || n > cap - p.E) { wrong = true; n = max(0, min(n, cap)); }
    int g = -1, pre = 0;
    if (p.n_groups > 0 && ordered) {
      int lo = 0, hi = p.n_groups - 1;                 // the last group that starts at or before b
#pragma unroll 1
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.group_start[mid] <= b) lo = mid; else hi = mid - 1;
      }
      g = lo;
      pre = p.prefix_len[g];
      if (pre < 0 || pre > n) { pl.bad[g] = 1; wrong = true; pre = 0; }
      if (a8_members(p, g) < 2) { g = -1; pre = 0; }   // nothing to share
    }
    pl.len[b] = n;
    pl.grp[b] = g;
    pl.pre[b] = pre;
  }
  wrong = __syncthreads_or(wrong || !ordered) != 0;
  if (wrong) {
#pragma unroll 1
    for (int b = tid; b < p.B; b += NT)
      if (pl.grp[b] >= 0 && pl.bad[pl.grp[b]]) { pl.grp[b] = -1; pl.pre[b] = 0; }
    if (tid == 0 && blockIdx.x == 0) sx_set_status(p.status, SX_ERR_CAPACITY);
    __syncthreads();
  }
  // exclusive sum of the units' list entries
  int run = 0;
#pragma unroll 1
  for (int u0 = 0; u0 < pl.units; u0 += NT) {
    const int u = u0 + tid;
    int x = 0;
    if (u < pl.units && (!PRE || ordered)) {
      const int st = a8_steps<PRE>(p, pl, ls, u, align);
      pl.steps[u] = st;
      x = st * p.nkv * a8_tiles(a8_unit_nq<PRE>(p, u), ls.qt_shift);
    }
    int s = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    if (lane == 31) wsum[warp] = s;
    __syncthreads();
    int before = run, all = 0;
#pragma unroll 1
    for (int w = 0; w < NT / 32; ++w) {
      const int y = wsum[w];
      if (w < warp) before += y;
      all += y;
    }
    if (u < pl.units) pl.cum[u] = before + s - x;
    run += all;
    __syncthreads();
  }
  if (tid == 0) pl.cum[pl.units] = run;
  pl.per = a8_per(run, ls);
  __syncthreads();
}

// what the merge needs to find the partial results again (CTA 0, once nothing earlier can still be reading it)
template <bool PRE, int NT>
__device__ __forceinline__ void a8_publish(const SxA8 &p, const A8Plan &pl, const SxA8List &ls) {
  if (blockIdx.x != 0) return;
#pragma unroll 1
  for (int u = threadIdx.x; u < pl.units; u += NT) {
    ls.cum[u] = pl.cum[u];
    ls.steps[u] = pl.cum[u + 1] > pl.cum[u] ? pl.steps[u] : 0;
  }
  if (threadIdx.x == 0) ls.total[0] = pl.cum[pl.units];
  if (!PRE)
#pragma unroll 1
    for (int b = threadIdx.x; b < p.B; b += NT) p.seq_group[b] = pl.pre[b] > 0 ? pl.grp[b] : -1;
}

// a place in a list: the segment (unit, head, tile) that holds list position x
struct A8Seg {
  int u, h, tile, cols;            // cols: queries of the tile
  int x0, x1;                      // list positions of the segment
  int b0, r0, first, end, len;     // table row, first query row, slots [first, end), cached slots
  int lo;                          // slots below it belong to the shared prefix
  int64_t base;                    // partial-result rows before qt * run is added
};
// (Written for few instructions: every role of the kernels that call it has a copy of it, and with divisions in 64 bits
// in here the code of a kernel passed 100 KB and ran out of the instruction cache: 14 us for the smallest call, and
// every part of the others several times slower.)
template <bool PRE>
__device__ __forceinline__ A8Seg a8_seek(const SxA8 &p, const A8Plan &pl, const SxA8List &ls, int align, int x) {
  A8Seg s;
  int lo = 0, hi = pl.units - 1;                       // the last unit that starts at or before x
#pragma unroll 1
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pl.cum[mid] <= x) lo = mid; else hi = mid - 1;
  }
  s.u = lo;
  const int nq = a8_unit_nq<PRE>(p, lo), nt = a8_tiles(nq, ls.qt_shift), steps = pl.steps[lo];
  const int r = (int)((uint32_t)(x - pl.cum[lo]) / (uint32_t)steps);
  s.h = nt == 1 ? r : (int)((uint32_t)r / (uint32_t)nt);
  s.tile = r - s.h * nt;
  s.cols = min(ls.qt, nq - (s.tile << ls.qt_shift));
  s.x0 = pl.cum[lo] + r * steps;
  s.x1 = s.x0 + steps;
  if (PRE) {
    s.b0 = p.group_start[lo];
    s.first = 0; s.lo = 0;
    s.end = pl.pre[s.b0]; s.len = s.end;
  } else {
    s.b0 = lo;
    s.lo = pl.pre[lo];
    s.first = s.lo & ~(align - 1);
    s.len = pl.len[lo]; s.end = min(s.len + p.E, p.max_pages * p.page);
  }
  s.r0 = s.b0 * p.rows;
  s.base = (int64_t)s.r0 * p.G * p.nkv + (int64_t)s.h * nq + (s.tile << ls.qt_shift);
  return s;
}
// bit j: slot first + j (j < n <= 32) is seen by a row of the segment whose drafted slots are `mask`
template <bool PRE>
__device__ __forceinline__ uint32_t a8_visible(const A8Seg &s, uint64_t mask, int first, int n) {
  const int a = max(s.lo - first, 0), b = min(s.len - first, n);
  uint64_t v = b > a ? ((1ull << b) - 1ull) & ~((1ull << a) - 1ull) : 0ull;
  if (!PRE) {
    const int drafted = s.end - s.len, at = first - s.len;        // drafted slots; position of `first` among them
    if (drafted < 64) mask &= (1ull << max(drafted, 0)) - 1ull;
    if (at >= 0) v |= at < 64 ? mask >> at : 0ull;
    else if (at > -32) v |= mask << -at;
  }
  return (uint32_t)v;
}

// The warp-level kernel's running softmax in base 2 is over s' = s + e, where 2^e is the scale of the slot's value row: the
// weight of a code row is 2^(s' - ref) and the weight of the slot itself 2^(s' - ref - e).  So the value scales cost no
// multiplication of V, and what is rounded (the weight) is the part that meets the codes, relative to the largest
// contribution: the largest code of a row is above 224, unless its scale is the smallest there is or the row is all
// zeros, which the kernel looks for.
__device__ __forceinline__ float a8_pow2(int byte) { return __uint_as_float((uint32_t)byte << 23); }        // 2^(byte - 127)
__device__ __forceinline__ float a8_pow2_inv(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
__device__ __forceinline__ float a8_exponent(int byte) {       // 255 marks a row with a value that is not finite
  return byte == 255 ? __int_as_float(0x7fffffff) : (float)(byte - 127);
}

// A pair of query values, scaled so that their row's largest magnitude lies in (224, 448], as pairs of e4m3 (high part) and
// e5m2 numbers (what is left).  A bf16 number has 8 significand bits; e4m3 keeps 4, and the rest is a multiple of the last
// bit, at most 8 of them: three significand bits, which e5m2 has, over a wider range.  So the sum is exact for values
// down to 2^-6, 2^-13 of the row's largest, and below that off by 2^-14 at most, 2^-21 of the largest (with e4m3 for both
// parts the exact range ended at 2^-10 of the largest and a value of 2^-12 of it was off by 1 %).
__device__ __forceinline__ void a8_split(float2 x, bool finite, uint32_t &hi, uint32_t &lo) {
  hi = (uint32_t)__nv_cvt_float2_to_fp8x2(x, __NV_SATFINITE, __NV_E4M3);
  const __half2_raw wide = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)hi, __NV_E4M3);
  const float2 back = __half22float2(*reinterpret_cast<const __half2 *>(&wide));
  lo = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x.x - back.x, x.y - back.y), __NV_SATFINITE, __NV_E5M2);
  if (!finite) hi = lo = 0x7f7fu;                      // a number in neither
}

size_t sx_attn8_ws_bytes(int nq, int nkv, int d, int B, int rows, int groups, int sm_count);
sx_status sx_launch_attn8_tc(const SxA8 &p, bool prefix, int sm_count, cudaStream_t st);
bool sx_attn8_tc_supported(const SxA8 &p);
sx_status sx_attn8_params(const sx_kv_shape &sh, const sx_kv &kv, int rows, int E, SxA8 *out);
sx_status sx_attn8_check(SxA8 p, int kernel, int sm_count);      // what sx_launch_attn8 would refuse
sx_status sx_launch_attn8(SxA8 p, int kernel, char *ws, int sm_count, cudaStream_t st);
