// Rotary positions: queries and keys turned to their positions, and rows turned on their way into a paged cache.
//
// Pair i of a head's rotated part turns by the angle pos * f_i:
//     (u, v) -> a (u cos - v sin, v cos + u sin),      transposed: sin -> -sin
// with u, v = x[i], x[i + r/2] (half order) or x[2i], x[2i + 1] (interleaved).  What has to be exact is the angle modulo one
// turn: in fp32 a position of 10^5 alone costs it 0.01 rad.  The plan keeps f_i / 2 pi as a 64-bit fraction of a turn, so
// that pos * f_i modulo one turn is one 64-bit integer product, whatever the position (off by pos * 2^-64 turns); its
// quadrant is taken off as an integer too, and what is left, at most an eighth of a turn, is small enough for a short series.  cos,
// sin and the products are fp32, of the angle's upper 32 bits (cut off at 2^-32 turns, 1.5e-9 rad, a fortieth of what fp32 makes of
// a cosine); fp64, of all 64, for keys that become codes.  The result is rounded once.
//
// Bound by bytes: every element is read and written once, three flops on the way.  A row (a head of a token) belongs to
// d / 8 neighbouring lanes with 8 elements each, 16-byte accesses; the partner half comes from another lane by shuffle,
// never a second time from memory.  A warp keeps the cos and sin of its lanes' elements in registers and takes a slice of a
// token's rows (all of them in large calls, down to one row per lane in small ones, where the latency of a wave is all
// there is).  64 registers, so that 32 warps of an SM have four rows each on the way.
//
// Measured (bf16, d = 128): 8192 tokens of 40 heads 29.9 us (168 MB, 5.6 TB/s; 55 us with 154 registers and the rows of all parts in
// one loop), 32 tokens 3.7 us.  Prompts of 34k tokens into bf16 pages, 32 query and 8 KV heads, 135 us (840 MB, 6.2 TB/s); one
// token of 32 sequences 4.5 us; 4096 tokens of keys (half of each turned) and values into an 8-bit cache 12.6 us (25 MB), bound by the
// conversions to and from fp64, four a clock and scheduler (10.2 us with fp32).
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "sx_kernels.cuh"
#include "sx_launch.cuh"

#define ROPE_THREADS 128

enum { PARTNER_LANE = 0, PARTNER_SHUFFLE = 1, PARTNER_LOAD = 2 };

struct SxRopeArgs {
  int T, D, nq, nk, nv;          // tokens; elements of a head; rows of a token: queries, keys, values
  int rot_start, rot_dim, half;  // half: 0 = interleaved order
  int partner;                   // where a lane finds the other half of its pairs, PARTNER_*
  int rows_per_warp, slices;
  double magnitude;
  int transpose;
  const int32_t *pos;            // [T] positions of the rows; append: nullptr = the row's slot
  const void *q, *k, *v;
  void *qo, *ko;                 // ko: rotation alone
  int64_t qs, ks, vs, qos, kos;
  // append alone
  int B, page, max_pages, num_pages;
  const int32_t *row_start, *pos_start, *page_table;
  void *kp, *vp;
  uint8_t *ksc, *vsc;
  int32_t *status;
};

struct SxRopeSteps { uint64_t step[SX_ROPE_MAX_PAIRS]; };

// magnitude * (cos, sin) of pos * step, step in 2^-64 turns.  After the quadrant is taken off, |x| <= pi / 4 and the Taylor
// series to x^9 and x^10 are off by 2e-9 and 1e-10 at most, below the roundings of their evaluation.
__device__ __forceinline__ void rope_angle(uint64_t step, int pos, double mag, float *c, float *s) {
  const float magnitude = (float)mag;
  const uint64_t ph = step * (uint64_t)(int64_t)pos;
  const uint32_t hi = (uint32_t)(ph >> 32), quad = (hi + (1u << 29)) >> 30;
  const float x = (float)(int32_t)(hi - (quad << 30)) * 1.4629180792671596e-9f;      // 2 pi / 2^32
  const float z = x * x;
  float sn = fmaf(z, 2.7557319223985893e-6f, -1.9841269841269841e-4f);
  sn = fmaf(z, sn, 8.3333333333333333e-3f);
  sn = fmaf(z, sn, -1.6666666666666667e-1f);
  sn = fmaf(z * x, sn, x);
  float cs = fmaf(z, -2.7557319223985891e-7f, 2.4801587301587302e-5f);
  cs = fmaf(z, cs, -1.3888888888888889e-3f);
  cs = fmaf(z, cs, 4.1666666666666667e-2f);
  cs = fmaf(z, cs, -0.5f);
  cs = fmaf(z, cs, 1.0f);
  const float u = (quad & 1) ? -sn : cs, v = (quad & 1) ? cs : sn;
  *c = magnitude * ((quad & 2) ? -u : u);
  *s = magnitude * ((quad & 2) ? -v : v);
}

// The same with all 64 bits of the angle, for rows that are going to be rounded to codes (see rope_turn): the series to x^13 and x^12 are
// off by 2^-45 and 2^-41 at most.
__device__ __forceinline__ void rope_angle(uint64_t step, int pos, double magnitude, double *c, double *s) {
  const uint64_t ph = step * (uint64_t)(int64_t)pos;
  const uint32_t quad = (uint32_t)((ph + (1ull << 61)) >> 62);
  const double x = (double)(int64_t)(ph - ((uint64_t)quad << 62)) * 3.4061215800304563e-19;      // 2 pi / 2^64
  const double z = x * x;
  double sn = fma(z, 1.6059043836821613e-10, -2.5052108385441720e-8);
  sn = fma(z, sn, 2.7557319223985893e-6);
  sn = fma(z, sn, -1.9841269841269841e-4);
  sn = fma(z, sn, 8.3333333333333332e-3);
  sn = fma(z, sn, -1.6666666666666666e-1);
  sn = fma(z * x, sn, x);
  double cs = fma(z, 2.0876756987868099e-9, -2.7557319223985888e-7);
  cs = fma(z, cs, 2.4801587301587302e-5);
  cs = fma(z, cs, -1.3888888888888889e-3);
  cs = fma(z, cs, 4.1666666666666664e-2);
  cs = fma(z, cs, -0.5);
  cs = fma(z, cs, 1.0);
  const double u = (quad & 1) ? -sn : cs, v = (quad & 1) ? cs : sn;
  *c = magnitude * ((quad & 2) ? -u : u);
  *s = magnitude * ((quad & 2) ? -v : v);
}

template <typename E> struct Rope8;                     // eight elements as words, and one element from memory
template <> struct Rope8<bf16> {
  enum { W = 4 };
  static __device__ __forceinline__ void unpack(const uint32_t *w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint32_t pack(const float *x, int i) {
    const __nv_bfloat162 y = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    return *reinterpret_cast<const uint32_t *>(&y);
  }
  static __device__ __forceinline__ float one(const bf16 *p) { return __bfloat162float(*p); }
};
template <> struct Rope8<__half> {
  enum { W = 4 };
  static __device__ __forceinline__ void unpack(const uint32_t *w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint32_t pack(const float *x, int i) {
    const __half2 y = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    return *reinterpret_cast<const uint32_t *>(&y);
  }
  static __device__ __forceinline__ float one(const __half *p) { return __half2float(*p); }
};
template <> struct Rope8<float> {
  enum { W = 8 };
  static __device__ __forceinline__ void unpack(const uint32_t *w, float *x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ uint32_t pack(const float *x, int i) { return __float_as_uint(x[i]); }
  static __device__ __forceinline__ float one(const float *p) { return *p; }
};

// What a lane needs for its eight elements of every row of one position.
template <typename F>
struct RopeLane {
  F c[8], s[8];                  // cos, and the signed sine that the partner is multiplied by
  uint32_t in;                   // bit e: element e is in the rotated part
  int src;                       // PARTNER_SHUFFLE: lane of the partner's elements
};

template <int PARTNER, typename F>
__device__ __forceinline__ void rope_lane_set(const SxRopeArgs &p, int e0, int lane, RopeLane<F> *r) {
  r->in = 0;
  r->src = lane;
#pragma unroll
  for (int e = 0; e < 8; ++e) r->c[e] = r->s[e] = F(0);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if ((unsigned)(e0 + e - p.rot_start) < (unsigned)p.rot_dim) r->in |= 1u << e;
  if (PARTNER == PARTNER_SHUFFLE && r->in) r->src = e0 - p.rot_start < p.half ? lane + p.half / 8 : lane - p.half / 8;
}

// Every lane of the warp calls it (shuffles).
template <int PARTNER, typename F>
__device__ __forceinline__ void rope_lane_angles(const SxRopeArgs &p, const SxRopeSteps &st, int e0, int pos, RopeLane<F> *r) {
  const int i0 = e0 - p.rot_start;
  if (PARTNER == PARTNER_LANE) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      F c = F(0), s = F(0);
      if (r->in >> e & 1) rope_angle(st.step[(i0 + e) >> 1], pos, p.magnitude, &c, &s);
      if (p.transpose) s = -s;
      r->c[e] = r->c[e + 1] = c;
      r->s[e] = -s;
      r->s[e + 1] = s;
    }
  } else if (PARTNER == PARTNER_SHUFFLE) {
    // both halves of the eight pairs turn by the same angles: the lane of the first half computes four, its partner the others
    const bool first = i0 < p.half;
    const uint64_t *step = st.step + (r->in ? (first ? i0 : i0 - p.half + 4) : 0);
    F c[4], s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) rope_angle(step[e], pos, p.magnitude, &c[e], &s[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const F oc = __shfl_sync(0xffffffffu, c[e], r->src), os = __shfl_sync(0xffffffffu, s[e], r->src);
      r->c[e] = first ? c[e] : oc;
      r->c[e + 4] = first ? oc : c[e];
      const bool minus = first != (p.transpose != 0);
      const F lo = first ? s[e] : os, hi = first ? os : s[e];
      r->s[e] = minus ? -lo : lo;
      r->s[e + 4] = minus ? -hi : hi;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      F c = F(0), s = F(0);
      const int i = i0 + e;
      if (r->in >> e & 1) rope_angle(st.step[i < p.half ? i : i - p.half], pos, p.magnitude, &c, &s);
      r->c[e] = c;
      r->s[e] = ((i < p.half) != (p.transpose != 0)) ? -s : s;
    }
  }
}

// To be rounded once more to fewer bits: cut off, with the last bit set if anything was lost, so that the second rounding is right.
__device__ __forceinline__ float rope_narrow(float y) { return y; }
__device__ __forceinline__ float rope_narrow(double y) {
  const float f = __double2float_rz(y);                       // loses the lower 29 bits of the fraction (more only below 2^-126)
  return (__double2loint(y) & 0x1fffffff) && fabsf(f) < INFINITY ? __uint_as_float(__float_as_uint(f) | 1u) : f;
}

// One row's words turned in place.  Every lane of the warp calls it (shuffles); row: nullptr where the lane has none.
// F = double where the row goes into codes: of a value within an fp32 rounding of the border between two of them the other code, a
// sixteenth of the value away, would be written (4096 tokens of 8 heads: some three values, 1e-4 of the result's norm).
template <typename E, int PARTNER, typename F>
__device__ __forceinline__ void rope_turn(const SxRopeArgs &p, const RopeLane<F> &r, const E *row, int e0, uint32_t *w) {
  constexpr int W = Rope8<E>::W;
  float x[8], o[8];
  Rope8<E>::unpack(w, x);
  if (PARTNER == PARTNER_LANE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = x[e ^ 1];
  } else if (PARTNER == PARTNER_SHUFFLE) {
    uint32_t ow[W];
#pragma unroll
    for (int i = 0; i < W; ++i) ow[i] = __shfl_sync(0xffffffffu, w[i], r.src);
    Rope8<E>::unpack(ow, o);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = e0 + e - p.rot_start;
      o[e] = (row && (r.in >> e & 1)) ? Rope8<E>::one(row + (i < p.half ? p.half : -p.half) + e0 + e) : 0.f;
    }
  }
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = rope_narrow(fma(F(x[e]), r.c[e], F(o[e]) * r.s[e]));
  // a word outside the rotated part keeps its bits (the part begins and ends between 32-bit words)
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const uint32_t m = 0u - (r.in >> (PARTNER == PARTNER_SHUFFLE ? 0 : i * (8 / W)) & 1u);
    w[i] = (w[i] & ~m) | (Rope8<E>::pack(y, i) & m);
  }
}

template <int W>
__device__ __forceinline__ void rope_load(const void *src, uint32_t *w) {
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    const uint4 v = reinterpret_cast<const uint4 *>(src)[i / 4];
    w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
  }
}
template <int W>
__device__ __forceinline__ void rope_store(void *dst, const uint32_t *w) {
#pragma unroll
  for (int i = 0; i < W; i += 4) reinterpret_cast<uint4 *>(dst)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
}

// Rows [h0, h1) of a token's queries or keys, G at a time, U times that on the way together.  angles() is called once the
// first rows have been asked for.
template <typename E, int LPR, int PARTNER, typename A>
__device__ __forceinline__ void rope_rows(const SxRopeArgs &p, RopeLane<float> &rl, int h0, int h1, const E *src, E *dst, int lane, A angles) {
  constexpr int W = Rope8<E>::W, G = 32 / LPR, U = PARTNER == PARTNER_LOAD ? 2 : 16 / W;
  const int e0 = (lane % LPR) * 8;
#pragma unroll 1
  for (int r = h0; r < h1; r += G * U) {
    uint32_t w[U][W];
    const int h = r + lane / LPR;
    const E *from = src + (int64_t)h * p.D + e0;
    E *to = dst + (int64_t)h * p.D + e0;
    const int n = e0 < p.D ? (h1 - h + G - 1) / G : 0;           // rows that this lane has
#pragma unroll
    for (int i = 0; i < U; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[i][j] = 0;
      if (i < n) rope_load<W>(from + i * G * p.D, w[i]);
    }
    angles();
#pragma unroll
    for (int i = 0; i < U; ++i) rope_turn<E, PARTNER>(p, rl, i < n ? from + i * G * p.D - e0 : nullptr, e0, w[i]);
    __syncwarp();                                   // in place: all of a row is read before any of it is written
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i < n) rope_store<W>(to + i * G * p.D, w[i]);
  }
}

// LPR lanes per row: the power of two from d / 8 up, at least 4
template <typename E, int LPR, int PARTNER>
__global__ void __launch_bounds__(ROPE_THREADS, PARTNER == PARTNER_LOAD ? 4 : 8) sx_rope_kernel(const SxRopeArgs p, const __grid_constant__ SxRopeSteps st) {
  sx_pdl_wait();
  const int lane = threadIdx.x & 31, unit = blockIdx.x * (ROPE_THREADS / 32) + (threadIdx.x >> 5);
  const int t = unit / p.slices;
  if (t >= p.T) return;
  const int r0 = (unit - t * p.slices) * p.rows_per_warp, r1 = min(p.nq + p.nk, r0 + p.rows_per_warp);
  const int e0 = (lane % LPR) * 8, pos = p.pos[t];
  RopeLane<float> rl;
  rope_lane_set<PARTNER>(p, e0, lane, &rl);
  bool set = false;
  const auto angles = [&]() {
    if (!set) rope_lane_angles<PARTNER>(p, st, e0, pos, &rl);
    set = true;
  };
  rope_rows<E, LPR, PARTNER>(p, rl, r0, min(r1, p.nq), reinterpret_cast<const E *>(p.q) + t * p.qs, reinterpret_cast<E *>(p.qo) + t * p.qos, lane, angles);
  rope_rows<E, LPR, PARTNER>(p, rl, max(r0 - p.nq, 0), r1 - p.nq, reinterpret_cast<const E *>(p.k) + t * p.ks, reinterpret_cast<E *>(p.ko) + t * p.kos, lane, angles);
}

// The sequence of row t (the last one that starts at or before it), found by the whole warp 32 at a time; -1: none.
__device__ __forceinline__ int rope_sequence(const SxRopeArgs &p, int t, int lane, int *first) {
  int lo = 0, n = p.B;
  while (true) {
    const int step = (n + 31) / 32, at = lane * step;
    const int s = at < n ? p.row_start[lo + at] : 0x7fffffff;
    const uint32_t m = __ballot_sync(0xffffffffu, s <= t);
    if (m == 0) return -1;
    const int h = 31 - __clz(m);
    *first = __shfl_sync(0xffffffffu, s, h);
    lo += h * step;
    n = min(step, n - h * step);
    if (step == 1) break;
  }
  return t < p.row_start[lo + 1] ? lo : -1;
}

// Rows [h0, h1) of a token's keys (TURN) or values to their places in the pool; Q8: as e4m3 codes with one power-of-two scale
// per row, as the unrotated append writes the exact rotation's row rounded to bf16.
template <int LPR, int PARTNER, bool Q8, bool TURN, typename F, typename A>
__device__ __forceinline__ void rope_place(const SxRopeArgs &p, RopeLane<F> &rl, int h0, int h1, const bf16 *src, void *pool, uint8_t *scales,
                                           const int64_t &place, int lane, A angles) {
  constexpr int G = 32 / LPR, U = PARTNER == PARTNER_LOAD ? 2 : 4;
  const int e0 = (lane % LPR) * 8;
#pragma unroll 1
  for (int r = h0; r < h1; r += G * U) {
    uint32_t w[U][4];
    const int h = r + lane / LPR;
    const bf16 *from = src + (int64_t)h * p.D + e0;
    int n = e0 < p.D ? (h1 - h + G - 1) / G : 0;                 // rows that this lane has
#pragma unroll
    for (int i = 0; i < U; ++i) {
      w[i][0] = w[i][1] = w[i][2] = w[i][3] = 0;
      if (i < n) rope_load<4>(from + i * G * p.D, w[i]);
    }
    angles();
    if (TURN) {
#pragma unroll
      for (int i = 0; i < U; ++i) rope_turn<bf16, PARTNER>(p, rl, i < n ? from + i * G * p.D - e0 : nullptr, e0, w[i]);
    }
    if (place < 0) n = 0;
    int64_t at = place + (int64_t)h * p.page;
#pragma unroll
    for (int i = 0; i < U; ++i, at += G * p.page) {
      if (Q8) {
        const uint32_t m = 0x7fff7fffu;
        uint32_t top = __vmaxu2(__vmaxu2(w[i][0] & m, w[i][1] & m), __vmaxu2(w[i][2] & m, w[i][3] & m));
        top = max(top & 0xffffu, top >> 16);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (i < n) {
          const int byte = sx_kv8_scale_byte(top);
          const float up = sx_kv8_inverse(byte);
          uint2 c = make_uint2(0, 0);
          if (byte != 255) c = make_uint2(sx_kv8_codes4(w[i][0], w[i][1], up), sx_kv8_codes4(w[i][2], w[i][3], up));
          *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(pool) + at * p.D + e0) = c;
          if (e0 == 0) scales[at] = (uint8_t)byte;
        }
      } else if (i < n) {
        rope_store<4>(reinterpret_cast<bf16 *>(pool) + at * p.D + e0, w[i]);
      }
    }
  }
}

// Rows of new tokens: queries and keys turned, keys and values to their pages.
template <int LPR, int PARTNER, bool Q8>
__global__ void __launch_bounds__(ROPE_THREADS, PARTNER == PARTNER_LOAD ? 4 : Q8 ? 7 : 8) sx_rope_append_kernel(const SxRopeArgs p, const __grid_constant__ SxRopeSteps st) {
  sx_pdl_wait();                              // dependents start when this kernel has completed: they may read the pages
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < p.B; b += ROPE_THREADS) {
      const int s = p.row_start[b], e = p.row_start[b + 1];
      if (s < 0 || e < s || e > p.T) sx_set_status(p.status, SX_ERR_CAPACITY);
    }
  const int lane = threadIdx.x & 31, unit = blockIdx.x * (ROPE_THREADS / 32) + (threadIdx.x >> 5);
  const int t = unit / p.slices;
  if (t >= p.T) return;
  const int r0 = (unit - t * p.slices) * p.rows_per_warp, r1 = min(p.nq + p.nk + p.nv, r0 + p.rows_per_warp);
  const int e0 = (lane % LPR) * 8;
  int first = 0;
  const int b = rope_sequence(p, t, lane, &first);
  if (b < 0) return;                          // a row behind the last sequence
  RopeLane<float> rl;
  rope_lane_set<PARTNER>(p, e0, lane, &rl);
  int64_t place = -1;                         // first row of the pool for this token
  int pos = 0;
  bool set = false;
  const auto find = [&]() {                   // while the first rows are on their way: the token's place and position
    if (set) return;
    set = true;
    const int64_t slot = (int64_t)p.pos_start[b] + (t - first), lp = slot < 0 ? -1 : slot / p.page;
    int pp = -1;
    if (lp >= 0 && lp < p.max_pages) pp = p.page_table[(int64_t)b * p.max_pages + lp];
    pos = p.pos ? p.pos[t] : (int)slot;
    if (pp < 0 || pp >= p.num_pages) sx_set_status(p.status, SX_ERR_CAPACITY);
    else place = (int64_t)pp * p.nk * p.page + slot % p.page;
  };
  const int k0 = p.nq, v0 = p.nq + p.nk;
  const bf16 *q = reinterpret_cast<const bf16 *>(p.q) + t * p.qs, *k = reinterpret_cast<const bf16 *>(p.k) + t * p.ks,
             *v = reinterpret_cast<const bf16 *>(p.v) + t * p.vs;
  bool turned = false;
  const auto angles = [&]() {
    find();
    if (!turned) rope_lane_angles<PARTNER>(p, st, e0, pos, &rl);
    turned = true;
  };
  rope_rows<bf16, LPR, PARTNER>(p, rl, r0, min(r1, k0), q, reinterpret_cast<bf16 *>(p.qo) + t * p.qos, lane, angles);
  const int k_from = max(r0 - k0, 0), k_to = min(r1, v0) - k0;
  if constexpr (Q8) {
    RopeLane<double> wide;
    rope_lane_set<PARTNER>(p, e0, lane, &wide);
    bool wide_set = false;
    rope_place<LPR, PARTNER, Q8, true>(p, wide, k_from, k_to, k, p.kp, p.ksc, place, lane, [&]() {
      find();
      if (!wide_set) rope_lane_angles<PARTNER>(p, st, e0, pos, &wide);
      wide_set = true;
    });
  } else {
    rope_place<LPR, PARTNER, Q8, true>(p, rl, k_from, k_to, k, p.kp, p.ksc, place, lane, angles);
  }
  rope_place<LPR, PARTNER, Q8, false>(p, rl, max(r0 - v0, 0), r1 - v0, v, p.vp, p.vsc, place, lane, find);
}

// ---- host side -----------------------------------------------------------------------------------------------------
extern "C" sx_status sx_rope_plan(const sx_rope_cfg *cfg, sx_rotation *out) {
  if (!cfg || !out) return SX_ERR_INVALID_ARG;
  const int r = cfg->rot_dim, d = cfg->head_dim, n = r / 2;
  if (d < 8 || d > SX_ROPE_MAX_HEAD || d % 8) return SX_ERR_UNSUPPORTED;
  if (r < 2 || r % 2 || cfg->rot_start < 0 || cfg->rot_start % 2 || cfg->rot_start > d - r) return SX_ERR_INVALID_ARG;
  if (cfg->layout != SX_ROPE_HALF && cfg->layout != SX_ROPE_INTERLEAVED) return SX_ERR_INVALID_ARG;
  const auto positive = [](double x) { return x > 0.0 && x < INFINITY; };
  if (!positive(cfg->theta) || !positive(cfg->magnitude) || !positive((double)(float)cfg->magnitude)) return SX_ERR_INVALID_ARG;
  if (cfg->scaling < SX_ROPE_NONE || cfg->scaling > SX_ROPE_LIST) return SX_ERR_INVALID_ARG;
  if (cfg->scaling != SX_ROPE_NONE && cfg->scaling != SX_ROPE_LIST && !positive(cfg->factor)) return SX_ERR_INVALID_ARG;
  if (cfg->scaling == SX_ROPE_BASE && r == 2) return SX_ERR_INVALID_ARG;
  const bool trained = cfg->scaling == SX_ROPE_BANDS || cfg->scaling == SX_ROPE_RAMP;
  if (trained && (!positive(cfg->low) || !positive(cfg->high) || cfg->low >= cfg->high || cfg->original_len < 1)) return SX_ERR_INVALID_ARG;
  if (cfg->scaling == SX_ROPE_RAMP && cfg->theta <= 1.0) return SX_ERR_INVALID_ARG;
  if (cfg->scaling == SX_ROPE_LIST) {
    if (!cfg->divisors) return SX_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i)
      if (!positive(cfg->divisors[i])) return SX_ERR_INVALID_ARG;
  }
  const long double TURN = 6.283185307179586476925286766559005768L, factor = cfg->factor;
  long double theta = cfg->theta, lo = 0, hi = 0;
  if (cfg->scaling == SX_ROPE_BASE) theta *= powl(factor, (long double)r / (r - 2));
  if (cfg->scaling == SX_ROPE_RAMP) {
    const long double per = r / (2.0L * logl(theta)), trained_turns = cfg->original_len / TURN;
    lo = fmaxl(floorl(per * logl(trained_turns / cfg->high)), 0.0L);
    hi = fminl(ceill(per * logl(trained_turns / cfg->low)), r - 1.0L);
  }
  memset(out, 0, sizeof(*out));
  for (int i = 0; i < n; ++i) {
    long double f = powl(theta, -2.0L * i / r), w;
    switch (cfg->scaling) {
      case SX_ROPE_LINEAR: f /= factor; break;
      case SX_ROPE_LIST: f /= cfg->divisors[i]; break;
      case SX_ROPE_BANDS:
        w = fminl(1.0L, fmaxl(0.0L, (cfg->original_len * f / TURN - cfg->low) / ((long double)cfg->high - cfg->low)));
        f *= w + (1.0L - w) / factor;
        break;
      case SX_ROPE_RAMP:
        w = fminl(1.0L, fmaxl(0.0L, (i - lo) / fmaxl(hi - lo, 1e-3L)));
        f *= 1.0L - w + w / factor;
        break;
      default: break;
    }
    long double turns = f / TURN;
    turns -= floorl(turns);
    const long double fixed = roundl(turns * 18446744073709551616.0L);
    if (!(fixed >= 0.0L)) return SX_ERR_INVALID_ARG;                   // a frequency beyond the range of a long double
    out->step[i] = fixed >= 18446744073709551616.0L ? 0 : (uint64_t)fixed;
  }
  out->head_dim = d;
  out->rot_start = cfg->rot_start;
  out->rot_dim = r;
  out->layout = cfg->layout;
  out->magnitude = cfg->magnitude;
  out->ready = SX_ROPE_READY;
  return SX_OK;
}

static bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }

// the plan's part of the arguments; a null plan turns nothing
static sx_status rope_args(const sx_rotation *plan, int head_dim, SxRopeArgs *p, SxRopeSteps *st) {
  memset(p, 0, sizeof(*p));
  memset(st, 0, sizeof(*st));
  p->D = head_dim;
  p->partner = PARTNER_LANE;
  if (!plan) return SX_OK;
  if (plan->ready != SX_ROPE_READY || plan->head_dim != head_dim || plan->rot_dim < 2 || plan->rot_start < 0 ||
      plan->rot_dim > head_dim - plan->rot_start || plan->rot_dim / 2 > SX_ROPE_MAX_PAIRS)
    return SX_ERR_INVALID_ARG;
  p->rot_start = plan->rot_start;
  p->rot_dim = plan->rot_dim;
  p->magnitude = plan->magnitude;
  if (plan->layout == SX_ROPE_HALF) {
    p->half = plan->rot_dim / 2;
    // halves that do not begin where a lane does: the partners come from memory one by one (8192 tokens of 40 heads with 120 of
    // 128 elements turned 56 us, with 112 by shuffle 30 us)
    p->partner = (p->half % 8 == 0 && p->rot_start % 8 == 0) ? PARTNER_SHUFFLE : PARTNER_LOAD;
  }
  memcpy(st->step, plan->step, sizeof(uint64_t) * (plan->rot_dim / 2));
  return SX_OK;
}

static int lanes_per_row(int d) { int l = 4; while (l * 8 < d) l <<= 1; return l; }

// A warp takes all rows of a token where that makes 16 warps per SM; below that the rows are cut into as many slices as make
// them, down to one row per lane (4, 8, 16, 32, 64 warps per SM: 512 tokens of 40 heads 6.1, 5.7, 5.3, 7.4, 7.8 us; 2048 of them the same
// within a tenth).
static sx_status rope_grid(SxRopeArgs *p, unsigned *grid) {
  if (p->T > 0x7ffffff0) return SX_ERR_UNSUPPORTED;                    // warps are counted in 32 bits
  const int all = p->nq + p->nk + p->nv, G = 32 / lanes_per_row(p->D);
  const int sm = sx_sm_count();
  if (!sm) return SX_ERR_CUDA;
  int slices = 1 + (16 * sm - 1) / p->T, most = (all + G - 1) / G;     // 16 sm / T rounded up
  if (slices > most) slices = most;
  p->rows_per_warp = ((all + slices - 1) / slices + G - 1) / G * G;
  p->slices = (all + p->rows_per_warp - 1) / p->rows_per_warp;
  const int64_t ctas = ((int64_t)p->T * p->slices + ROPE_THREADS / 32 - 1) / (ROPE_THREADS / 32);
  if ((int64_t)p->T * p->slices > 0x7ffffff0ll) return SX_ERR_UNSUPPORTED;
  *grid = (unsigned)ctas;
  return SX_OK;
}

template <typename E, int PARTNER>
static sx_status launch_rope_of(const SxRopeArgs &p, const SxRopeSteps &s, unsigned grid, cudaStream_t st) {
  switch (lanes_per_row(p.D)) {
    case 4: return sx_rc(sx_launch(sx_rope_kernel<E, 4, PARTNER>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
    case 8: return sx_rc(sx_launch(sx_rope_kernel<E, 8, PARTNER>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
    case 16: return sx_rc(sx_launch(sx_rope_kernel<E, 16, PARTNER>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
    default: return sx_rc(sx_launch(sx_rope_kernel<E, 32, PARTNER>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
  }
}
template <typename E>
static sx_status launch_rope(const SxRopeArgs &p, const SxRopeSteps &s, unsigned grid, cudaStream_t st) {
  if (p.partner == PARTNER_LANE) return launch_rope_of<E, PARTNER_LANE>(p, s, grid, st);
  if (p.partner == PARTNER_SHUFFLE) return launch_rope_of<E, PARTNER_SHUFFLE>(p, s, grid, st);
  return launch_rope_of<E, PARTNER_LOAD>(p, s, grid, st);
}

extern "C" sx_status sx_rope(const sx_rotation *plan, int32_t dtype, int32_t transpose, int32_t T, const int32_t *pos_d,
                             int32_t n_q, const void *q_d, int64_t q_stride, void *q_out_d, int64_t q_out_stride, int32_t n_k,
                             const void *k_d, int64_t k_stride, void *k_out_d, int64_t k_out_stride, void *stream) {
  if (!plan || dtype < SX_BF16 || dtype > SX_F32 || T < 0 || n_q < 0 || n_k < 0 || (transpose != 0 && transpose != 1)) return SX_ERR_INVALID_ARG;
  if (n_q > SX_ROPE_MAX_ROWS || n_k > SX_ROPE_MAX_ROWS) return SX_ERR_UNSUPPORTED;
  SxRopeArgs p;
  SxRopeSteps s;
  SX_TRY(rope_args(plan, plan->head_dim, &p, &s));
  const int64_t lanes = dtype == SX_F32 ? 4 : 8;                       // elements of a 16-byte access
  const auto part = [&](int32_t n, const void *x, int64_t xs, const void *y, int64_t ys) {
    if (n == 0) return true;
    const int64_t row = (int64_t)n * p.D;
    return aligned16(x) && aligned16(y) && xs >= row && ys >= row && xs % lanes == 0 && ys % lanes == 0 && (x != y || xs == ys);
  };
  if (!part(n_q, q_d, q_stride, q_out_d, q_out_stride) || !part(n_k, k_d, k_stride, k_out_d, k_out_stride)) return SX_ERR_INVALID_ARG;
  if (T == 0 || n_q + n_k == 0) return SX_OK;
  if (!pos_d) return SX_ERR_INVALID_ARG;
  p.T = T; p.nq = n_q; p.nk = n_k; p.pos = pos_d; p.transpose = transpose;
  p.q = q_d; p.k = k_d; p.qo = q_out_d; p.ko = k_out_d;
  p.qs = q_stride; p.ks = k_stride; p.qos = q_out_stride; p.kos = k_out_stride;
  unsigned grid;
  SX_TRY(rope_grid(&p, &grid));
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == SX_BF16) return launch_rope<bf16>(p, s, grid, st);
  if (dtype == SX_F16) return launch_rope<__half>(p, s, grid, st);
  return launch_rope<float>(p, s, grid, st);
}

template <bool Q8, int PARTNER>
static sx_status launch_append_of(const SxRopeArgs &p, const SxRopeSteps &s, unsigned grid, cudaStream_t st) {
  switch (lanes_per_row(p.D)) {
    case 4: return sx_rc(sx_launch(sx_rope_append_kernel<4, PARTNER, Q8>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
    case 8: return sx_rc(sx_launch(sx_rope_append_kernel<8, PARTNER, Q8>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
    default: return sx_rc(sx_launch(sx_rope_append_kernel<16, PARTNER, Q8>, dim3(grid), dim3(ROPE_THREADS), 0, st, p, s));
  }
}
template <bool Q8>
static sx_status launch_append(const SxRopeArgs &p, const SxRopeSteps &s, unsigned grid, cudaStream_t st) {
  if (p.partner == PARTNER_LANE) return launch_append_of<Q8, PARTNER_LANE>(p, s, grid, st);
  if (p.partner == PARTNER_SHUFFLE) return launch_append_of<Q8, PARTNER_SHUFFLE>(p, s, grid, st);
  return launch_append_of<Q8, PARTNER_LOAD>(p, s, grid, st);
}

extern "C" sx_status sx_kv_append_rope(const sx_rotation *plan, const sx_kv_shape *sh, const sx_kv *kv, int32_t T,
                                       const int32_t *row_start_d, const int32_t *pos_start_d, const int32_t *rot_pos_d,
                                       const void *k_d, int64_t k_stride, const void *v_d, int64_t v_stride, const void *q_d,
                                       int64_t q_stride, void *q_out_d, int64_t q_out_stride, int32_t *status_d, void *stream) {
  SX_TRY(sx_kv_check_cache(sh, kv));
  const int d = sh->head_dim;
  if (d != 16 && d != 32 && d != 64 && d != 128) return SX_ERR_UNSUPPORTED;
  if (T < 0 || !row_start_d || !status_d || !aligned16(k_d) || !aligned16(v_d)) return SX_ERR_INVALID_ARG;
  const int64_t row = (int64_t)sh->n_kv_heads * d;
  if (k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8) return SX_ERR_INVALID_ARG;
  if (sh->n_kv_heads > SX_ROPE_MAX_ROWS || sh->n_q_heads > SX_ROPE_MAX_ROWS) return SX_ERR_UNSUPPORTED;
  SxRopeArgs p;
  SxRopeSteps s;
  SX_TRY(rope_args(plan, d, &p, &s));
  if (q_d || q_out_d) {
    const int64_t qrow = (int64_t)sh->n_q_heads * d;
    if (sh->n_q_heads < 1 || !aligned16(q_d) || !aligned16(q_out_d) || q_stride < qrow || q_out_stride < qrow || q_stride % 8 ||
        q_out_stride % 8 || (q_d == q_out_d && q_stride != q_out_stride))
      return SX_ERR_INVALID_ARG;
    p.nq = sh->n_q_heads;
    p.q = q_d; p.qo = q_out_d; p.qs = q_stride; p.qos = q_out_stride;
  }
  if (T == 0) return SX_OK;
  p.T = T; p.nk = p.nv = sh->n_kv_heads;
  p.pos = rot_pos_d;
  p.k = k_d; p.v = v_d; p.ks = k_stride; p.vs = v_stride;
  p.B = kv->batch; p.page = sh->page_size; p.max_pages = kv->max_pages; p.num_pages = kv->num_pages;
  p.row_start = row_start_d; p.pos_start = pos_start_d ? pos_start_d : kv->cache_len_d; p.page_table = kv->page_table_d;
  p.kp = kv->k_pages_d; p.vp = kv->v_pages_d;
  p.status = status_d;
  unsigned grid;
  SX_TRY(rope_grid(&p, &grid));
  if (kv->dtype == SX_KV_E4M3) {
    p.ksc = kv->k_scale_d; p.vsc = kv->v_scale_d;
    return launch_append<true>(p, s, grid, (cudaStream_t)stream);
  }
  return launch_append<false>(p, s, grid, (cudaStream_t)stream);
}
