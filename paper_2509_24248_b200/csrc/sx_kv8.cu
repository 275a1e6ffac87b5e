// The 8-bit paged KV cache: writing rows into it and reading them back, and the entry points of the operators over it.
//
// A row is one token of one KV head, x[0..d) in bf16.  Its scale is the power of two 2^e with
//     e = ceil(log2(max |x| / 448)), held to [-64, 120]; 0 for a row of zeros,   stored as the byte e + 127,
// and its codes are e4m3(x * 2^-e), round to nearest even.  448 = 1.75 * 2^8 is the largest e4m3 value, so e follows from
// the exponent and the top of the mantissa of max |x| alone, x * 2^-e is exact, and a code times its scale is exact in
// bf16 again (but for values from 248 * 2^120 up, which round to 2^128): nothing but the rounding to 4 significand bits happens, the same on every path that writes a row.  A row
// with a value that is not finite gets the byte 255 and codes of zero; readers turn the byte into NaN.
//
// Both kernels are bound by bytes: 4 d + 2 d + 2 per token and head.  A CTA takes a few consecutive rows of the
// token buffer (a token's K row is contiguous), finds sequence and page of each once, and moves 16 bytes per
// thread: d / 8 lanes share a row when writing, so the maximum is a few shuffles; d / 16 when reading.  Measured with 8 heads
// of 128: 34k tokens written in 51 us (210 MB, 4.1 TB/s, 68 % of the issue slots), 140k read in 172 us (867 MB, 5.0 TB/s),
// one token of 32 sequences written in 4.5 us.  (Tried: rows in the order of the pages rather than of the buffer when
// writing, 81 against 63 us; stores past the cache when reading, 218 against 197 us.)
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "sx_attn8.cuh"
#include "sx_kernels.cuh"
#include "sx_launch.cuh"

#define KV8_THREADS 256
#define KV8_MAX_TOKENS 64            // tokens per CTA

struct SxKv8Rows {
  int B, T, nkv, d, page, max_pages, num_pages, tokens;      // tokens: per CTA
  const int32_t *row_start, *pos_start, *page_table;
  int64_t k_stride, v_stride;
  uint8_t *k, *v, *ks, *vs;
  int32_t *status;
};

// First row of the pool (page * n_kv * page_size + offset, to which head * page_size is added) of the CTA's tokens, -1
// where there is no token.  Every thread looks at some sequences and names the tokens that belong to them; then a
// thread per token finds its page.
__device__ __forceinline__ void kv8_places(const SxKv8Rows &p, int t0, int nt, int64_t *place) {
  __shared__ int seq[KV8_MAX_TOKENS];
  for (int i = threadIdx.x; i < nt; i += KV8_THREADS) seq[i] = -1;
  __syncthreads();
#pragma unroll 1
  for (int b = threadIdx.x; b < p.B; b += KV8_THREADS) {
    const int s = p.row_start[b], e = p.row_start[b + 1];
    if (blockIdx.x == 0 && (s < 0 || e < s || e > p.T)) sx_set_status(p.status, SX_ERR_CAPACITY);
    for (int t = max(max(s, 0), t0); t < min(e, t0 + nt); ++t) seq[t - t0] = b;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nt; i += KV8_THREADS) {
    const int b = seq[i];
    int64_t at = -1;
    if (b >= 0) {
      const int64_t pos = (int64_t)p.pos_start[b] + (t0 + i - p.row_start[b]), lp = pos < 0 ? -1 : pos / p.page;
      int pp = -1;
      if (lp >= 0 && lp < p.max_pages) pp = p.page_table[(int64_t)b * p.max_pages + lp];
      if (pp < 0 || pp >= p.num_pages) sx_set_status(p.status, SX_ERR_CAPACITY);
      else at = (int64_t)pp * p.nkv * p.page + pos % p.page;
    }
    place[i] = at;
  }
  __syncthreads();
}

template <int D>
__global__ void __launch_bounds__(KV8_THREADS) sx_kv8_append_kernel(SxKv8Rows p, const bf16 *__restrict__ k, const bf16 *__restrict__ v) {
  constexpr int LPR = D / 8;
  __shared__ int64_t place[KV8_MAX_TOKENS];
  sx_pdl_wait();                              // dependents start when this kernel has completed: they may read the pages
  const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.T - t0);
  kv8_places(p, t0, nt, place);
  const int rows = nt * p.nkv * 2, lane = threadIdx.x % LPR;
  // row index: token, K or V, head.  Four rows per thread at a time, so that their loads are on the way together.
  constexpr int U = 4, RPC = KV8_THREADS / LPR;
  const int per = 2 * p.nkv;                 // rows of a token: its heads' keys, then their values
  int t_at = (int)(threadIdx.x / LPR) / per, w_at = (int)(threadIdx.x / LPR) - t_at * per;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += U * RPC) {
    uint4 x[U];
    int64_t at[U];
    bool is_v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int t = t_at, h = w_at < p.nkv ? w_at : w_at - p.nkv;
      is_v[i] = w_at >= p.nkv;
      at[i] = t < nt ? place[t] : -1;
      w_at += RPC;
      while (w_at >= per) { w_at -= per; ++t_at; }
      x[i] = make_uint4(0, 0, 0, 0);
      if (at[i] >= 0) {
        at[i] += (int64_t)h * p.page;
        const bf16 *src = is_v[i] ? v + (int64_t)(t0 + t) * p.v_stride : k + (int64_t)(t0 + t) * p.k_stride;
        x[i] = *reinterpret_cast<const uint4 *>(src + (int64_t)h * D + lane * 8);
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t m = 0x7fff7fffu;
      uint32_t top = __vmaxu2(__vmaxu2(x[i].x & m, x[i].y & m), __vmaxu2(x[i].z & m, x[i].w & m));
      top = max(top & 0xffffu, top >> 16);
#pragma unroll
      for (int o = 1; o < LPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int byte = sx_kv8_scale_byte(top);
      const float up = sx_kv8_inverse(byte);
      uint2 c = make_uint2(0, 0);
      if (byte != 255) c = make_uint2(sx_kv8_codes4(x[i].x, x[i].y, up), sx_kv8_codes4(x[i].z, x[i].w, up));
      if (at[i] >= 0) {
        *reinterpret_cast<uint2 *>((is_v[i] ? p.v : p.k) + at[i] * D + lane * 8) = c;
        if (lane == 0) (is_v[i] ? p.vs : p.ks)[at[i]] = (uint8_t)byte;
      }
    }
  }
}

// U rows per thread at a time: eight in large calls (172 us against 197 us for 140k tokens of 8 heads), four in small ones
// (9.8 us against 13 us for 4096), where most of eight would not exist
template <int D, int U>
__global__ void __launch_bounds__(KV8_THREADS) sx_kv8_read_kernel(SxKv8Rows p, bf16 *__restrict__ k, bf16 *__restrict__ v) {
  constexpr int LPR = D / 16;
  __shared__ int64_t place[KV8_MAX_TOKENS];
  sx_pdl_wait();
  const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.T - t0);
  kv8_places(p, t0, nt, place);
  const int rows = nt * p.nkv * 2, lane = threadIdx.x % LPR;
  constexpr int RPC = KV8_THREADS / LPR;
  const int per = 2 * p.nkv;
  int w_at = (int)(threadIdx.x / LPR) / nt, t_at = (int)(threadIdx.x / LPR) - w_at * nt;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += U * RPC) {
    uint4 x[U];
    int byte[U];
    bf16 *dst[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int t = t_at, h = w_at < p.nkv ? w_at : w_at - p.nkv;
      const bool is_v = w_at >= p.nkv;
      dst[i] = nullptr;
      const bool on = w_at < per;
      t_at += RPC;
      while (t_at >= nt) { t_at -= nt; ++w_at; }
      if (on && place[t] >= 0) {
        const int64_t at = place[t] + (int64_t)h * p.page;
        x[i] = *reinterpret_cast<const uint4 *>((is_v ? p.v : p.k) + at * D + lane * 16);
        byte[i] = (is_v ? p.vs : p.ks)[at];
        dst[i] = (is_v ? v + (int64_t)(t0 + t) * p.v_stride : k + (int64_t)(t0 + t) * p.k_stride) + (int64_t)h * D + lane * 16;
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (!dst[i]) continue;
      const float s = byte[i] == 255 ? __int_as_float(0x7fffffff) : __uint_as_float((uint32_t)byte[i] << 23);
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint32_t o[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[q >> 1] >> ((q & 1) * 16)), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        const __nv_bfloat162 y = __floats2bfloat162_rn(f.x * s, f.y * s);
        o[q] = *reinterpret_cast<const uint32_t *>(&y);
      }
      reinterpret_cast<uint4 *>(dst[i])[0] = make_uint4(o[0], o[1], o[2], o[3]);
      reinterpret_cast<uint4 *>(dst[i])[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
  }
}

// ---- entry points ------------------------------------------------------------------------------------------------
static bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }

// a cache of either kind
sx_status sx_kv_check_cache(const sx_kv_shape *sh, const sx_kv *kv) {
  if (!sh || !kv || !kv->cache_len_d || !kv->page_table_d || !aligned16(kv->k_pages_d) || !aligned16(kv->v_pages_d))
    return SX_ERR_INVALID_ARG;
  if (kv->dtype != SX_KV_BF16 && kv->dtype != SX_KV_E4M3) return SX_ERR_UNSUPPORTED;
  if (kv->dtype == SX_KV_E4M3 && (!aligned16(kv->k_scale_d) || !aligned16(kv->v_scale_d))) return SX_ERR_INVALID_ARG;
  if (kv->batch < 1 || kv->max_pages < 1 || kv->num_pages < 1 || sh->n_kv_heads < 1 || sh->page_size < 1) return SX_ERR_INVALID_ARG;
  if (kv->dtype == SX_KV_E4M3 && sh->page_size % 16) return SX_ERR_UNSUPPORTED;
  if ((int64_t)kv->max_pages * sh->page_size > 0x7fffff00ll) return SX_ERR_UNSUPPORTED;     // slots are 32-bit
  return SX_OK;
}

static sx_status check_cache(const sx_kv_shape *sh, const sx_kv *kv) {
  SX_TRY(sx_kv_check_cache(sh, kv));
  return kv->dtype == SX_KV_E4M3 ? SX_OK : SX_ERR_UNSUPPORTED;
}

// SMs of the current device (asked for once per device), 0 on an error
int sx_sm_count() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

static sx_status rows_call(const sx_kv_shape *sh, const sx_kv *kv, int32_t T, const int32_t *row_start_d,
                           const int32_t *pos_start_d, const void *k, const void *v, int64_t ks, int64_t vs,
                           int32_t *status_d, SxKv8Rows *out) {
  SX_TRY(check_cache(sh, kv));
  const int d = sh->head_dim;
  if (d != 16 && d != 32 && d != 64 && d != 128) return SX_ERR_UNSUPPORTED;
  if (T < 0 || !row_start_d || !status_d || !aligned16(k) || !aligned16(v)) return SX_ERR_INVALID_ARG;
  const int64_t row = (int64_t)sh->n_kv_heads * d;
  if (ks < row || vs < row || ks % 8 || vs % 8) return SX_ERR_INVALID_ARG;
  SxKv8Rows p;
  memset(&p, 0, sizeof(p));
  p.B = kv->batch; p.T = T; p.nkv = sh->n_kv_heads; p.d = d; p.page = sh->page_size;
  p.max_pages = kv->max_pages; p.num_pages = kv->num_pages;
  p.row_start = row_start_d; p.pos_start = pos_start_d ? pos_start_d : kv->cache_len_d; p.page_table = kv->page_table_d;
  p.k_stride = ks; p.v_stride = vs;
  p.k = (uint8_t *)kv->k_pages_d; p.v = (uint8_t *)kv->v_pages_d; p.ks = kv->k_scale_d; p.vs = kv->v_scale_d;
  p.status = status_d;
  // as many tokens per CTA as make one wave of about six CTAs per SM: finding the places is a chain of three dependent
  // reads, which a CTA of few tokens spends half its time on
  const int wave = 6 * sx_sm_count();
  p.tokens = wave ? (T + wave - 1) / wave : 1;
  if (p.tokens > KV8_MAX_TOKENS) p.tokens = KV8_MAX_TOKENS;
  if (p.tokens < 1) p.tokens = 1;
  *out = p;
  return SX_OK;
}

extern "C" sx_status sx_kv_append(const sx_kv_shape *sh, const sx_kv *kv, int32_t T, const int32_t *row_start_d,
                                  const int32_t *pos_start_d, const void *k_d, int64_t k_stride, const void *v_d,
                                  int64_t v_stride, int32_t *status_d, void *stream) {
  SxKv8Rows p;
  SX_TRY(rows_call(sh, kv, T, row_start_d, pos_start_d, k_d, v_d, k_stride, v_stride, status_d, &p));
  if (T == 0) return SX_OK;
  const dim3 grid((T + p.tokens - 1) / p.tokens);
  const bf16 *k = (const bf16 *)k_d, *v = (const bf16 *)v_d;
  cudaStream_t st = (cudaStream_t)stream;
  switch (p.d) {
    case 16: return sx_rc(sx_launch(sx_kv8_append_kernel<16>, grid, dim3(KV8_THREADS), 0, st, p, k, v));
    case 32: return sx_rc(sx_launch(sx_kv8_append_kernel<32>, grid, dim3(KV8_THREADS), 0, st, p, k, v));
    case 64: return sx_rc(sx_launch(sx_kv8_append_kernel<64>, grid, dim3(KV8_THREADS), 0, st, p, k, v));
    default: return sx_rc(sx_launch(sx_kv8_append_kernel<128>, grid, dim3(KV8_THREADS), 0, st, p, k, v));
  }
}

template <int D>
static sx_status launch_read(const SxKv8Rows &p, dim3 grid, bf16 *k, bf16 *v, cudaStream_t st) {
  if (p.tokens < 16) return sx_rc(sx_launch(sx_kv8_read_kernel<D, 4>, grid, dim3(KV8_THREADS), 0, st, p, k, v));
  return sx_rc(sx_launch(sx_kv8_read_kernel<D, 8>, grid, dim3(KV8_THREADS), 0, st, p, k, v));
}

extern "C" sx_status sx_kv_read(const sx_kv_shape *sh, const sx_kv *kv, int32_t T, const int32_t *row_start_d,
                                const int32_t *pos_start_d, void *k_d, int64_t k_stride, void *v_d, int64_t v_stride,
                                int32_t *status_d, void *stream) {
  SxKv8Rows p;
  if (!pos_start_d) return SX_ERR_INVALID_ARG;
  SX_TRY(rows_call(sh, kv, T, row_start_d, pos_start_d, k_d, v_d, k_stride, v_stride, status_d, &p));
  if (T == 0) return SX_OK;
  const dim3 grid((T + p.tokens - 1) / p.tokens);
  bf16 *k = (bf16 *)k_d, *v = (bf16 *)v_d;
  cudaStream_t st = (cudaStream_t)stream;
  switch (p.d) {
    case 16: return launch_read<16>(p, grid, k, v, st);
    case 32: return launch_read<32>(p, grid, k, v, st);
    case 64: return launch_read<64>(p, grid, k, v, st);
    default: return launch_read<128>(p, grid, k, v, st);
  }
}

extern "C" size_t sx_attention_ws_bytes(const sx_kv_shape *sh, int32_t batch, int32_t rows, int32_t n_groups) {
  if (!sh || batch < 1 || rows < 1 || sh->n_q_heads < 1 || sh->head_dim < 1 || n_groups < 0) return 0;
  const int sm = sx_sm_count();
  return sm ? sx_attn8_ws_bytes(sh->n_q_heads, sh->n_kv_heads, sh->head_dim, batch, rows, n_groups, sm) : 0;
}

// the checks and the parameter block that the stand-alone call and the draft step share
sx_status sx_attn8_params(const sx_kv_shape &sh, const sx_kv &kv, int rows, int E, SxA8 *out) {
  SX_TRY(check_cache(&sh, &kv));
  if (sh.head_dim != 64 && sh.head_dim != 128) return SX_ERR_UNSUPPORTED;
  if (sh.n_q_heads < 1 || sh.n_q_heads % sh.n_kv_heads) return SX_ERR_UNSUPPORTED;
  if (rows < 1 || rows > SX_MAX_TREE_ROWS || E < 0 || E > SX_MAX_TREE_ROWS) return SX_ERR_INVALID_ARG;
  if (kv.n_groups < 0 || kv.n_groups > kv.batch) return SX_ERR_INVALID_ARG;
  if (kv.n_groups > 0 && (!kv.group_start_d || !kv.prefix_len_d)) return SX_ERR_INVALID_ARG;
  if (kv.batch + kv.n_groups > A8_MAX_UNITS || (int64_t)kv.batch * rows > 65535) return SX_ERR_UNSUPPORTED;
  SxA8 p;
  memset(&p, 0, sizeof(p));
  p.nq = sh.n_q_heads; p.nkv = sh.n_kv_heads; p.G = sh.n_q_heads / sh.n_kv_heads; p.d = sh.head_dim; p.page = sh.page_size;
  p.B = kv.batch; p.rows = rows; p.E = E; p.n_groups = kv.n_groups; p.max_pages = kv.max_pages; p.num_pages = kv.num_pages;
  p.cache_len = kv.cache_len_d; p.page_table = kv.page_table_d;
  p.group_start = kv.group_start_d; p.prefix_len = kv.prefix_len_d;
  p.k = (const uint8_t *)kv.k_pages_d; p.v = (const uint8_t *)kv.v_pages_d; p.ks = kv.k_scale_d; p.vs = kv.v_scale_d;
  *out = p;
  return SX_OK;
}

extern "C" sx_status sx_attention(const sx_kv_shape *sh, const sx_kv *kv, int32_t rows, int32_t drafted, const void *q_d,
                                  int64_t q_stride, const uint64_t *row_mask_d, float scale, int32_t kernel, void *o_d,
                                  void *ws_d, size_t ws_bytes, int32_t *status_d, void *stream) {
  if (!sh || !kv) return SX_ERR_INVALID_ARG;
  SxA8 p;
  SX_TRY(sx_attn8_params(*sh, *kv, rows, drafted, &p));
  if (!aligned16(q_d) || !aligned16(o_d) || !status_d || !(scale > -INFINITY && scale < INFINITY)) return SX_ERR_INVALID_ARG;
  if (kernel < SX_ATTN_AUTO || kernel > SX_ATTN_TC) return SX_ERR_INVALID_ARG;
  if (q_stride < (int64_t)p.nq * p.d || q_stride % 8) return SX_ERR_INVALID_ARG;
  const int sm = sx_sm_count();
  if (!sm) return SX_ERR_CUDA;
  if (!ws_d || ((uintptr_t)ws_d & 255) || ws_bytes < sx_attn8_ws_bytes(p.nq, p.nkv, p.d, p.B, rows, p.n_groups, sm))
    return SX_ERR_WORKSPACE;
  p.scale_log2 = (float)((double)scale * 1.4426950408889634);
  p.q_stride = q_stride;
  p.q = (const bf16 *)q_d;
  p.row_mask = row_mask_d;
  p.o_out = (bf16 *)o_d;
  p.status = status_d;
  return sx_launch_attn8(p, kernel, (char *)ws_d, sm, (cudaStream_t)stream);
}
