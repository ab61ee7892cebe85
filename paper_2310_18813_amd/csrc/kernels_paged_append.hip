// Keys and values of new rows into a paged cache, queries and keys rotated on the way (the rotary embedding of the models here:
// element i of a head turns with i + R/2 by the angle position * inv_freq[i]).
//
// One pass over q, k and v: 2 * rows * (Hq + 2 Hkv) * hd elements move, three operations a rotated element, so memory bounds it, and
// with few rows the chain length -> page -> store does.  4548 rows of 52 + 104 heads of 128, fp16: 74 us a call for 363 MB (4.9 TB/s); 256 rows
// of 32 + 16 heads, bf16: 3.7 us a call in a captured graph.
#include "paged.h"

namespace spec {

int paged_args(const char *who, const spec_paged_cache *c, const spec_paged_batch *b, PagedArgs *out) {
  if (!c || !b) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: cache or batch is null", who);
  if (c->dtype < SPEC_DTYPE_F32 || c->dtype > SPEC_DTYPE_F16) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: unknown dtype %d", who, c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128) return fail_noctx(SPEC_ERR_UNSUPPORTED, "%s: head_dim %d is neither 64 nor 128", who, c->head_dim);
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return fail_noctx(SPEC_ERR_UNSUPPORTED, "%s: page_size %d is not a power of two from 8 to 1024", who, c->page_size);
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->n_pages < 1)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: n_kv_heads=%d n_pages=%d", who, c->n_kv_heads, c->n_pages);
  const int64_t unit = 16 / (int64_t)dtype_bytes(c->dtype);
  const int64_t strides[3] = {c->page_stride, c->pos_stride, c->head_stride};
  for (int64_t s : strides)
    if (s < 0 || s % unit) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: cache strides must be non-negative multiples of 16 bytes", who);
  for (int64_t s : strides)
    if (s / unit > 0xffffffffll) return fail_noctx(SPEC_ERR_CAPACITY, "%s: a cache stride of 64 GB or more", who);
  if (c->pos_stride < c->head_dim || (c->n_kv_heads > 1 && c->head_stride < c->head_dim) || (c->n_pages > 1 && c->page_stride < c->head_dim))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: a cache stride is shorter than a head", who);
  if (!c->d_k || !c->d_v || ((uintptr_t)c->d_k & 15) || ((uintptr_t)c->d_v & 15))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: cache pointers must be set and 16-byte aligned", who);
  if (b->B < 0 || b->rows < 0) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: B=%d rows=%d", who, b->B, b->rows);
  if (b->B > 65535) return fail_noctx(SPEC_ERR_CAPACITY, "%s: at most 65535 sequences", who);
  if (b->B > 0 && b->rows > 0) {
    if (!b->d_len || !b->d_pages) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: d_len or d_pages is null", who);
    if (!b->d_row_start && b->rows % b->B) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: %d rows do not divide into %d sequences", who, b->rows, b->B);
    if (b->max_rows < 1 || b->max_rows > b->rows) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: max_rows=%d outside 1..%d", who, b->max_rows, b->rows);
    if (!b->d_row_start && b->max_rows < b->rows / b->B)
      return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: max_rows=%d, but every sequence brings %d", who, b->max_rows, b->rows / b->B);
    if (b->pages_stride < 1 || b->max_len < 1 || (int64_t)b->max_len > (int64_t)b->pages_stride * c->page_size)
      return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: max_len=%d outside 1..%d pages of %d", who, b->max_len, b->pages_stride, c->page_size);
    if (b->max_len > (1 << 30)) return fail_noctx(SPEC_ERR_CAPACITY, "%s: max_len=%d beyond 2^30", who, b->max_len);
  }
  *out = PagedArgs{(unsigned char *)c->d_k, (unsigned char *)c->d_v, (uint32_t)(c->page_stride / unit), (uint32_t)(c->pos_stride / unit),
                   (uint32_t)(c->head_stride / unit), c->n_pages,
                   __builtin_ctz(c->page_size), c->n_kv_heads, b->B, b->rows, b->max_rows, b->max_len, b->d_row_start, b->d_len, b->d_pages,
                   b->pages_stride};
  return SPEC_OK;
}

int paged_rows_check(const char *who, const char *what, const spec_paged_cache *c, int heads, const void *p, int64_t stride) {
  const int64_t unit = 16 / (int64_t)dtype_bytes(c->dtype);
  if (!p || ((uintptr_t)p & 15)) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: %s must be set and 16-byte aligned", who, what);
  if (stride < (int64_t)heads * c->head_dim || stride % unit)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: the row stride of %s must hold %d heads and be a multiple of 16 bytes", who, what, heads);
  return SPEC_OK;
}

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_v;

struct AppendArgs {
  PagedArgs p;
  const unsigned char *q, *k, *v;
  unsigned char *q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements
  const double *inv_freq;
  int n_q, half;  // query heads; half the rotated elements
};

// 16 bytes as numbers and back
template <class T> struct Unit {
  static constexpr int E = 16 / sizeof(T);
  static __device__ __forceinline__ void load(const u32x4_v &x, float (&f)[E]) {
    T t[E];
    __builtin_memcpy(t, &x, 16);
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = Conv<T>::ld(t, i);
  }
  static __device__ __forceinline__ u32x4_v store(const float (&f)[E]) {
    T t[E];
#pragma unroll
    for (int i = 0; i < E; ++i) Conv<T>::st(t, i, f[i]);
    u32x4_v x;
    __builtin_memcpy(&x, t, 16);
    return x;
  }
};

// The sequence of a row: how many sequences end at or before it.  A wave reads the boundaries together.
__device__ __forceinline__ int row_sequence(const PagedArgs &a, int row) {
  if (!a.row_start) return row / (a.rows / a.B);
  int b = 0;
  for (int k0 = 0; k0 < a.B; k0 += 64) {
    const int k = k0 + (int)(threadIdx.x & 63);
    const bool before = k < a.B && a.row_start[min(k, a.B - 1) + 1] <= row;
    b += __popcll(__ballot(before));
  }
  return b;
}

// A workgroup takes one row and 256 of its items; an item is two units of 16 bytes of a head: a rotated pair of them, or two that pass.
template <class T, int HD>
__global__ __launch_bounds__(256) void k_paged_append(AppendArgs a) {
  constexpr int E = Unit<T>::E, ITEMS = HD / (2 * E);
  __shared__ float2 turn[HD / 2];
  const int row = blockIdx.x;
  const int b = __builtin_amdgcn_readfirstlane(row_sequence(a.p, row));
  if (b >= a.p.B) return;
  const PagedSeq s = paged_seq(a.p, b);
  const int pos = s.kv - s.n + (row - s.row0);
  if (row < s.row0 || row - s.row0 >= s.n || pos < 0) return;
  const int page = paged_page(a.p, b, pos);
  if ((int)threadIdx.x < a.half) {
    // the angle in turns: what is left of it after whole turns is exact to 2^-32 of a turn for positions below 2^20
    const double turns = (double)pos * a.inv_freq[threadIdx.x] * 0.15915494309189533577;
    const float x = (float)(turns - rint(turns));
    float sn, cs;
    sincospif(2.f * x, &sn, &cs);
    turn[threadIdx.x] = make_float2(cs, sn);
  }
  __syncthreads();
  const int item = (int)blockIdx.y * 256 + (int)threadIdx.x, head = item / ITEMS, u = item % ITEMS;
  const int Hk = a.p.n_kv_heads;
  if (head >= a.n_q + 2 * Hk) return;
  const bool is_q = head < a.n_q, is_v = head >= a.n_q + Hk;
  const int h = is_q ? head : is_v ? head - a.n_q - Hk : head - a.n_q;
  const unsigned char *src = is_q ? a.q + (row * a.q_stride + h * HD) * sizeof(T)
                                  : is_v ? a.v + (row * a.v_stride + h * HD) * sizeof(T) : a.k + (row * a.k_stride + h * HD) * sizeof(T);
  unsigned char *dst;
  if (is_q) {
    dst = a.q_out + (row * a.q_out_stride + h * HD) * sizeof(T);
  } else {
    if (page < 0) return;
    dst = (is_v ? a.p.v : a.p.k) + paged_row(a.p, page, pos) + ((size_t)h * a.p.head_units << 4);
  }
  const int hu = a.half / E;  // units of a rotated half
  const bool turns = !is_v && u < hu;
  const int u0 = turns ? u : is_v ? 2 * u : 2 * u, u1 = turns ? u + hu : u0 + 1;
  u32x4_v x0 = ((const u32x4_v *)src)[u0], x1 = ((const u32x4_v *)src)[u1];
  if (turns) {
    float f0[E], f1[E];
    Unit<T>::load(x0, f0);
    Unit<T>::load(x1, f1);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float2 t = turn[u * E + i];
      const float y0 = f0[i] * t.x - f1[i] * t.y, y1 = f1[i] * t.x + f0[i] * t.y;
      f0[i] = y0; f1[i] = y1;
    }
    x0 = Unit<T>::store(f0);
    x1 = Unit<T>::store(f1);
  }
  ((u32x4_v *)dst)[u0] = x0;
  ((u32x4_v *)dst)[u1] = x1;
}

}  // namespace spec

using namespace spec;

extern "C" int spec_paged_append(void *hip_stream, const spec_paged_cache *cache, const spec_paged_batch *batch, int32_t n_q_heads,
                                 const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v,
                                 int64_t v_stride, const double *d_inv_freq, int32_t rope_dim, void *d_q_out, int64_t q_out_stride) {
  const char *who = "spec_paged_append";
  AppendArgs a{};
  int rc = paged_args(who, cache, batch, &a.p);
  if (rc) return rc;
  if (n_q_heads < 0 || n_q_heads > 65535) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: n_q_heads=%d", who, n_q_heads);
  if (rope_dim < 0 || rope_dim > cache->head_dim || rope_dim % 16)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: rope_dim=%d is not a multiple of 16 up to head_dim=%d", who, rope_dim, cache->head_dim);
  if (batch->B == 0 || batch->rows == 0) return SPEC_OK;
  if (rope_dim && !d_inv_freq) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: d_inv_freq is null", who);
  if (n_q_heads) {
    if ((rc = paged_rows_check(who, "d_q", cache, n_q_heads, d_q, q_stride))) return rc;
    if ((rc = paged_rows_check(who, "d_q_out", cache, n_q_heads, d_q_out, q_out_stride))) return rc;
    if (d_q == d_q_out && q_stride != q_out_stride)
      return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: rotation in place needs one row stride", who);
  }
  if ((rc = paged_rows_check(who, "d_k", cache, cache->n_kv_heads, d_k, k_stride))) return rc;
  if ((rc = paged_rows_check(who, "d_v", cache, cache->n_kv_heads, d_v, v_stride))) return rc;
  a.q = (const unsigned char *)d_q; a.k = (const unsigned char *)d_k; a.v = (const unsigned char *)d_v;
  a.q_out = (unsigned char *)d_q_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
  a.inv_freq = d_inv_freq; a.n_q = n_q_heads; a.half = rope_dim / 2;
  SPEC_DISPATCH_DTYPE(cache->dtype, T, {
    const int items = (n_q_heads + 2 * cache->n_kv_heads) * (cache->head_dim / (2 * Unit<T>::E));
    const dim3 grid(batch->rows, (items + 255) / 256);
    if ((int64_t)grid.x * grid.y * 256 >= (int64_t)1 << 32)
      return fail_noctx(SPEC_ERR_CAPACITY, "%s: %d rows of %d heads are beyond one launch", who, batch->rows, n_q_heads + 2 * cache->n_kv_heads);
    if (cache->head_dim == 64) hipLaunchKernelGGL((k_paged_append<T, 64>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
    else hipLaunchKernelGGL((k_paged_append<T, 128>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
