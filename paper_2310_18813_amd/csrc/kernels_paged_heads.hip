// Queries and keys normed per head and rotated on their way into a paged cache, of the rows' own type or of 8 bits, and a cache of 8 bits
// read back.
//
//   y = x / sqrt(mean(x^2) + eps) * w  (where there is a w),  then pairs of elements turn by position * inv_freq:  i with i + R/2, or
//   2i with 2i + 1.  Of 8 bits: code = e4m3(y / 2^e), e the smallest exponent with max |y| <= 448 * 2^e, one a position and key head.
//
// One pass over q, k and v; memory bounds it, and with few rows the chain length -> page -> store does.  A thread holds 16 or 8 elements of a
// head (two units of 16 bytes: whole pairs, whichever way they are paired), so that a head's sum and maximum are 2 to 4 exchanges between
// neighbouring lanes.  A key that becomes codes is computed in 64 bits: a value next to the border of two codes is then on the side where
// the definition has it, and what an append leaves does not depend on how it was computed.  Everything else is fp32 and rounded once.
// One row 3.4 us in a captured graph; 4553 rows of 52 + 104 heads of 128, fp16, normed, 364 MB: 78 us (4.7 TB/s, a copy's rate); 4530 rows of 32 + 64 into
// 8 bits, 186 MB: 46 (4.0 TB/s; keys in fp32 would take 41; 50 before the rows' loads went ahead of length and page; four items a thread 51); read
// back, 197 MB: 45 (4.4 TB/s).
#include "paged.h"
#include "paged8.h"
#include <cmath>

namespace spec {

struct HeadArgs {
  PagedArgs p;
  const unsigned char *q, *k, *v;
  unsigned char *q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements
  const double *inv_freq;
  const unsigned char *q_norm, *k_norm;
  double eps;
  int n_q, half, interleaved;  // query heads; half the rotated elements
};

// The value of a neighbour: lanes 1 and 2 apart, the other four of eight and the other eight of sixteen (mirrored, which is no matter once
// the nearer ones hold the same).
template <int CTRL> __device__ __forceinline__ int across(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <int CTRL> __device__ __forceinline__ double across(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)across<CTRL>((int)(uint32_t)u), hi = (uint32_t)across<CTRL>((int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL> __device__ __forceinline__ float across(float v) { return __int_as_float(across<CTRL>(__float_as_int(v))); }
template <int N, class V, class F> __device__ __forceinline__ V over_lanes(V v, F f) {  // N = 4, 8 or 16 neighbours
  v = f(v, across<0xb1>(v));
  v = f(v, across<0x4e>(v));
  if constexpr (N >= 8) v = f(v, across<0x141>(v));
  if constexpr (N >= 16) v = f(v, across<0x140>(v));
  return v;
}

// x: a thread's elements of a head; turn: (cosine, sine) of its pairs' angles
template <class A, class T2, int N>
__device__ __forceinline__ void rotate(A (&x)[N], const T2 *turn, bool interleaved) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const T2 t = turn[i];
    if (interleaved) {
      const A a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * t.x - b * t.y;
      x[2 * i + 1] = b * t.x + a * t.y;
    } else {
      const A a = x[i], b = x[N / 2 + i];
      x[i] = a * t.x - b * t.y;
      x[N / 2 + i] = b * t.x + a * t.y;
    }
  }
}

// A thread's 16 elements of a head as codes: two words each of its two units, and the exponent of the head's scale.
template <class T, int LANES>
__device__ __forceinline__ int encode(const float (&y)[16], uint2 &c0, uint2 &c1) {
  // A head that the rows' type cannot hold is NaN throughout (a maximum would lose a NaN: it becomes an infinity first).
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float m = fabsf(y[i]);
    top = fmaxf(top, m < Codes<T>::beyond ? m : INFINITY);
  }
  top = over_lanes<LANES>(top, [](float a, float b) { return fmaxf(a, b); });
  const bool odd = !(top < INFINITY);
  // top = m 2^x, m from 0.5 up to 1; 448 = 0.875 * 2^9
  int x;
  const float m = frexpf(top, &x);
  const int e = odd || !(top > 0.f) ? Codes<T>::least : max(Codes<T>::least, x - 9 + (m > 0.875f));
  float z[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = ldexpf(fminf(fmaxf(y[i], -Codes<T>::most), Codes<T>::most), -e);
  auto four = [&](int i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(z[i], z[i + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(z[i + 2], z[i + 3], w, true);
    return odd ? 0x7f7f7f7fu : (uint32_t)w;
  };
  c0 = make_uint2(four(0), four(4));
  c1 = make_uint2(four(8), four(12));
  return e;
}

// A workgroup takes one row and 256 of its items; an item is two units of 16 bytes of a head: rotated pairs, or elements that pass.
template <class T, int HD, bool C8>
__global__ __launch_bounds__(256) void k_paged_heads(HeadArgs a) {
  constexpr int E = Unit<T>::E, ITEMS = HD / (2 * E);
  __shared__ float2 turn[HD / 2];
  __shared__ double2 turn64[C8 ? HD / 2 : 1];
  const int row = blockIdx.x, item = (int)blockIdx.y * 256 + (int)threadIdx.x, head = item / ITEMS, u = item % ITEMS;
  const int Hk = a.p.n_kv_heads, hu = a.half / E;  // hu: items of a head that turn
  const bool on = head < a.n_q + 2 * Hk, is_q = head < a.n_q, is_v = head >= a.n_q + Hk;  // (on: all lanes of a head at once)
  const int h = is_q ? head : is_v ? head - a.n_q - Hk : head - a.n_q;
  const bool turns = !is_v && u < hu;
  const int u0 = turns && !a.interleaved ? u : 2 * u, u1 = turns && !a.interleaved ? u + hu : u0 + 1;
  // the loads first: whether anything comes of them takes three loads after one another, and the angles
  u32x4_v x0, x1;
  if (on) {
    const unsigned char *src = is_q ? a.q + (row * a.q_stride + h * HD) * sizeof(T)
                                    : is_v ? a.v + (row * a.v_stride + h * HD) * sizeof(T) : a.k + (row * a.k_stride + h * HD) * sizeof(T);
    x0 = ((const u32x4_v *)src)[u0];
    x1 = ((const u32x4_v *)src)[u1];
  }
  const int b = __builtin_amdgcn_readfirstlane(row_sequence(a.p, row));
  if (b >= a.p.B) return;
  const PagedSeq s = paged_seq(a.p, b);
  const int pos = s.kv - s.n + (row - s.row0);
  if (row < s.row0 || row - s.row0 >= s.n || pos < 0) return;
  const int page = paged_page(a.p, b, pos);
  if ((int)threadIdx.x < a.half) {
    // the angle in turns, of which whole ones are left out
    const double angle = (double)pos * a.inv_freq[threadIdx.x] * 0.15915494309189533577;
    const double part = angle - rint(angle);
    if (C8 && (int)(blockIdx.y * 256 + 255) / ITEMS >= a.n_q) {  // (queries alone do with fp32)
      double sn, cs;
      sincospi(2. * part, &sn, &cs);
      turn64[threadIdx.x] = make_double2(cs, sn);
      turn[threadIdx.x] = make_float2((float)cs, (float)sn);
    } else {
      float sn, cs;
      sincospif(2.f * (float)part, &sn, &cs);
      turn[threadIdx.x] = make_float2(cs, sn);
    }
  }
  __syncthreads();
  if (!on || (!is_q && page < 0)) return;
  const unsigned char *norm = is_q ? a.q_norm : is_v ? nullptr : a.k_norm;
  float x[2 * E], w[2 * E];
  auto unpack = [](const u32x4_v &lo, const u32x4_v &hi, float (&f)[2 * E]) {
    float f0[E], f1[E];
    Unit<T>::load(lo, f0);
    Unit<T>::load(hi, f1);
#pragma unroll
    for (int i = 0; i < E; ++i) { f[i] = f0[i]; f[E + i] = f1[i]; }
  };
  unpack(x0, x1, x);
  double r = 1.;
  if (norm) {
    unpack(((const u32x4_v *)norm)[u0], ((const u32x4_v *)norm)[u1], w);
    double ss = 0.;  // (squares of large bf16 values leave fp32)
#pragma unroll
    for (int i = 0; i < 2 * E; ++i) ss = fma((double)x[i], (double)x[i], ss);
    ss = over_lanes<ITEMS>(ss, [](double p, double q) { return p + q; });
    r = 1. / sqrt(ss * (1. / HD) + a.eps);
  }
  if constexpr (C8) {
    if (!is_q) {
      uint2 c0, c1;
      int e;
      if (is_v) {
        e = encode<T, ITEMS>(x, c0, c1);
      } else {
        double y[2 * E];
#pragma unroll
        for (int i = 0; i < 2 * E; ++i) y[i] = norm ? (double)x[i] * r * (double)w[i] : (double)x[i];
        if (turns) rotate(y, turn64 + u * E, a.interleaved);
        // To 32 bits so that codes and scales come out as from 64: they ask for nothing but on which side of numbers of a few bits a value lies.
        float z[2 * E];
#pragma unroll
        for (int i = 0; i < 2 * E; ++i) z[i] = to_odd(y[i]);
        e = encode<T, ITEMS>(z, c0, c1);
      }
      unsigned char *dst = (is_v ? a.p.v : a.p.k) + paged_row(a.p, page, pos) + ((size_t)h * a.p.head_units << 4);
      if (u1 == u0 + 1) {  // (units beside each other: all but half pairs)
        ((uint4 *)dst)[u0 >> 1] = make_uint4(c0.x, c0.y, c1.x, c1.y);
      } else {
        ((uint2 *)dst)[u0] = c0;
        ((uint2 *)dst)[u1] = c1;
      }
      if (u == 0) (is_v ? a.p.v_scale : a.p.k_scale)[paged_scale(a.p, page, h, pos)] = (uint8_t)(e + 127);
      return;
    }
  }
  unsigned char *dst = is_q ? a.q_out + (row * a.q_out_stride + h * HD) * sizeof(T)
                            : (is_v ? a.p.v : a.p.k) + paged_row(a.p, page, pos) + ((size_t)h * a.p.head_units << 4);
  u32x4_v y0 = x0, y1 = x1;
  if (norm || turns) {
    if (norm) {
      // (r itself leaves fp32 where x and eps are small)
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) x[i] = (float)((double)x[i] * r) * w[i];
    }
    if (turns) rotate(x, turn + u * E, a.interleaved);
    float f0[E], f1[E];
#pragma unroll
    for (int i = 0; i < E; ++i) { f0[i] = x[i]; f1[i] = x[E + i]; }
    y0 = Unit<T>::store(f0);
    y1 = Unit<T>::store(f1);
  }
  ((u32x4_v *)dst)[u0] = y0;
  ((u32x4_v *)dst)[u1] = y1;
}

struct ReadArgs {
  PagedArgs p;
  unsigned char *k, *v;
  int64_t k_stride, v_stride;  // elements
};

// A thread takes 16 elements of a head.
template <class T, int HD>
__global__ __launch_bounds__(256) void k_paged8_read(ReadArgs a) {
  constexpr int ITEMS = HD / 16;
  const int row = blockIdx.x;
  const int b = __builtin_amdgcn_readfirstlane(row_sequence(a.p, row));
  if (b >= a.p.B) return;
  const PagedSeq s = paged_seq(a.p, b);
  const int pos = s.kv - s.n + (row - s.row0);
  if (row < s.row0 || row - s.row0 >= s.n || pos < 0) return;
  const int page = paged_page(a.p, b, pos);
  const int item = (int)blockIdx.y * 256 + (int)threadIdx.x, head = item / ITEMS, u = item % ITEMS;
  const int Hk = a.p.n_kv_heads;
  if (head >= 2 * Hk) return;
  const bool is_v = head >= Hk;
  const int h = is_v ? head - Hk : head;
  unsigned char *dst = is_v ? a.v : a.k;
  if (!dst) return;
  dst += (row * (is_v ? a.v_stride : a.k_stride) + h * HD + 16 * u) * sizeof(T);
  u32x4_v y0 = {0, 0, 0, 0}, y1 = y0;
  if (page >= 0) {
    const u32x4_v c = ((const u32x4_v *)((is_v ? a.p.v : a.p.k) + paged_row(a.p, page, pos) + ((size_t)h * a.p.head_units << 4)))[u];
    const float scale = scale_of((is_v ? a.p.v_scale : a.p.k_scale)[paged_scale(a.p, page, h, pos)]);
    decode16<T>(c, scale, y0, y1);
  }
  ((u32x4_v *)dst)[0] = y0;
  ((u32x4_v *)dst)[1] = y1;
}

static int heads_check(const char *who, const spec_paged_cache *c, const spec_paged_batch *b, const spec_head_transform *t, int n_q, const void *d_q,
                       int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride, void *d_q_out, int64_t q_out_stride,
                       HeadArgs &a) {
  static const spec_head_transform none = {nullptr, 0, 0, nullptr, nullptr, 0.};
  if (!t) t = &none;
  int rc;
  if (n_q < 0 || n_q > 65535) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: n_q_heads=%d", who, n_q);
  if (t->rope_dim < 0 || t->rope_dim > c->head_dim || t->rope_dim % 16)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: rope_dim=%d is not a multiple of 16 up to head_dim=%d", who, t->rope_dim, c->head_dim);
  if (t->interleaved != 0 && t->interleaved != 1) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: interleaved=%d is neither 0 nor 1", who, t->interleaved);
  if ((t->d_q_norm || t->d_k_norm) && !(t->eps > 0. && t->eps < INFINITY))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: norms need a positive eps", who);
  if (((uintptr_t)t->d_q_norm & 15) || ((uintptr_t)t->d_k_norm & 15))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: the norms' weights must be 16-byte aligned", who);
  if (b->B == 0 || b->rows == 0) return SPEC_OK;
  if (t->rope_dim && !t->d_inv_freq) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: d_inv_freq is null", who);
  if (n_q) {
    if ((rc = paged_rows_check(who, "d_q", c, n_q, d_q, q_stride))) return rc;
    if ((rc = paged_rows_check(who, "d_q_out", c, n_q, d_q_out, q_out_stride))) return rc;
    if (d_q == d_q_out && q_stride != q_out_stride)
      return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: rotation in place needs one row stride", who);
  }
  if ((rc = paged_rows_check(who, "d_k", c, c->n_kv_heads, d_k, k_stride))) return rc;
  if ((rc = paged_rows_check(who, "d_v", c, c->n_kv_heads, d_v, v_stride))) return rc;
  a.q = (const unsigned char *)d_q; a.k = (const unsigned char *)d_k; a.v = (const unsigned char *)d_v;
  a.q_out = (unsigned char *)d_q_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
  a.inv_freq = t->d_inv_freq; a.n_q = n_q; a.half = t->rope_dim / 2; a.interleaved = t->interleaved;
  a.q_norm = (const unsigned char *)t->d_q_norm; a.k_norm = (const unsigned char *)t->d_k_norm; a.eps = t->eps;
  return SPEC_OK;
}

template <bool C8>
static int heads_launch(const char *who, const spec_paged_cache *c, int rows, const HeadArgs &a, hipStream_t st) {
  SPEC_DISPATCH_DTYPE(c->dtype, T, {
    if constexpr (!C8 || sizeof(T) == 2) {
      const int items = (a.n_q + 2 * c->n_kv_heads) * (c->head_dim / (2 * Unit<T>::E));
      const dim3 grid(rows, (items + 255) / 256);
      if ((int64_t)grid.x * grid.y * 256 >= (int64_t)1 << 32)
        return fail_noctx(SPEC_ERR_CAPACITY, "%s: %d rows of %d heads are beyond one launch", who, rows, a.n_q + 2 * c->n_kv_heads);
      if (c->head_dim == 64) hipLaunchKernelGGL((k_paged_heads<T, 64, C8>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((k_paged_heads<T, 128, C8>), grid, dim3(256), 0, st, a);
    }
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}

}  // namespace spec

using namespace spec;

extern "C" int spec_paged_append_normed(void *hip_stream, const spec_paged_cache *cache, const spec_paged_batch *batch,
                                        const spec_head_transform *transform, int32_t n_q_heads, const void *d_q, int64_t q_stride, const void *d_k,
                                        int64_t k_stride, const void *d_v, int64_t v_stride, void *d_q_out, int64_t q_out_stride) {
  const char *who = "spec_paged_append_normed";
  HeadArgs a{};
  int rc = paged_args(who, cache, batch, &a.p);
  if (!rc) rc = heads_check(who, cache, batch, transform, n_q_heads, d_q, q_stride, d_k, k_stride, d_v, v_stride, d_q_out, q_out_stride, a);
  if (rc || batch->B == 0 || batch->rows == 0) return rc;
  return heads_launch<false>(who, cache, batch->rows, a, (hipStream_t)hip_stream);
}

extern "C" int spec_paged8_append(void *hip_stream, const spec_paged_cache8 *cache, const spec_paged_batch *batch,
                                  const spec_head_transform *transform, int32_t n_q_heads, const void *d_q, int64_t q_stride, const void *d_k,
                                  int64_t k_stride, const void *d_v, int64_t v_stride, void *d_q_out, int64_t q_out_stride) {
  const char *who = "spec_paged8_append";
  HeadArgs a{};
  spec_paged_cache as;
  int rc = paged8_args(who, cache, batch, &as, &a.p);
  if (!rc) rc = heads_check(who, &as, batch, transform, n_q_heads, d_q, q_stride, d_k, k_stride, d_v, v_stride, d_q_out, q_out_stride, a);
  if (rc || batch->B == 0 || batch->rows == 0) return rc;
  return heads_launch<true>(who, &as, batch->rows, a, (hipStream_t)hip_stream);
}

extern "C" int spec_paged8_read(void *hip_stream, const spec_paged_cache8 *cache, const spec_paged_batch *batch, void *d_k, int64_t k_stride,
                                void *d_v, int64_t v_stride) {
  const char *who = "spec_paged8_read";
  ReadArgs a{};
  spec_paged_cache as;
  int rc = paged8_args(who, cache, batch, &as, &a.p);
  if (rc || batch->B == 0 || batch->rows == 0) return rc;
  if (!d_k && !d_v) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: d_k and d_v are null", who);
  if (d_k && (rc = paged_rows_check(who, "d_k", &as, as.n_kv_heads, d_k, k_stride))) return rc;
  if (d_v && (rc = paged_rows_check(who, "d_v", &as, as.n_kv_heads, d_v, v_stride))) return rc;
  a.k = (unsigned char *)d_k; a.v = (unsigned char *)d_v;
  a.k_stride = k_stride; a.v_stride = v_stride;
  const int items = 2 * as.n_kv_heads * (as.head_dim / 16);
  const dim3 grid(batch->rows, (items + 255) / 256);
  if ((int64_t)grid.x * grid.y * 256 >= (int64_t)1 << 32)
    return fail_noctx(SPEC_ERR_CAPACITY, "%s: %d rows of %d heads are beyond one launch", who, batch->rows, 2 * as.n_kv_heads);
  hipStream_t st = (hipStream_t)hip_stream;
  if (as.dtype == SPEC_DTYPE_BF16) hipLaunchKernelGGL((as.head_dim == 64 ? k_paged8_read<bf16_t, 64> : k_paged8_read<bf16_t, 128>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((as.head_dim == 64 ? k_paged8_read<f16_t, 64> : k_paged8_read<f16_t, 128>), grid, dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
