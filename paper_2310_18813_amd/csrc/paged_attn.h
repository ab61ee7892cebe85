// Attention of new rows over a paged cache, causal, with grouped heads and an optional sliding window.
//
//   out[row, h] = sum_k w_k V[k, h / G],  w = softmax over the visible k of scale * q[row, h] . K[k, h / G]
//
// The rows of a sequence and the G query heads of a key head are one list of n * G query rows that share every cached row: tile t of it
// is the query rows t * R .. t * R + R - 1.  A workgroup takes one tile, one key head and one chunk of the tile's positions; its four
// waves take every fourth step of 32 positions.  One pass with a running maximum and sum; what several chunks leave is joined by a
// second kernel.  Transposed as in the verification attention of the contexts, so that no score moves between lanes:
//   S^T[key][query] = K . Q^T,   O^T[dim][query] += V^T . P^T
// The first product's result layout (lane = query, 4 keys a lane and tile) is the second's operand layout once row 4g + i of key tile t
// carries key 8g + 4t + i.  Keys come from memory in operand order; of values a lane loads the same 8 or 4 elements of 8
// positions, whole rows of a head across 16 lanes, and turns the block round in registers.
// Few rows are bound by their loads: 64 sequences x 4 rows of 32 heads of 128 over up to 1000 positions, bf16, 650 MB in 125 us
// (5.2 TB/s), and the loads without any arithmetic took as long.  Six sequences of up to 32000 positions, 32 heads over 8: 102 us.
// The same over 8 bits, 329 MB: 74 us (4.4 TB/s; the loads without arithmetic 70).
//
// S, what the cache holds: the rows' type T, or e4m3 codes, which become numbers of T times their scale (exactly) on the way to the products:
// keys and values of few rows in registers, those of many rows on their way to LDS.
//
// Chunks: a sequence with more rows or positions has more work, and the host does not know the lengths.  Every wave adds the
// batch's work up (a load and a few ALU instructions) and cuts it by what an even share would be, whatever the lengths are.
#pragma once
#include "paged8.h"
#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

namespace spec {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_v;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_v;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_v;
typedef __attribute__((ext_vector_type(2))) float f32x2_v;
typedef __attribute__((ext_vector_type(4))) float f32x4_v;

constexpr int PA_CHUNK_MIN = 512; // positions of the shortest chunk
constexpr int PA_WAVES = 4;

struct AttendArgs {
  PagedArgs p;
  const unsigned char *q;
  unsigned char *out;
  int64_t q_stride, out_stride;  // elements
  int G, window;
  float sl2;                     // scale * log2(e)
  float *part, *ml;              // partial results of tiles that are cut: [part * heads][R][HD], [part * heads][R][2]
  int chunk_min;
  float one_slot;                // 1 / workgroups per key head that the work is cut into
};

// ------------------------------------------------------------------ work
struct Work { int b, tile, chunk, chunks, chunk_len, part; PagedSeq s; };

// Sums over the lanes of a wave up to each lane, in a few ALU instructions (a shuffle goes through LDS, and every workgroup starts with this).
template <int CTRL, int ROWS> __device__ __forceinline__ int from_lane(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int sum_to(int v) {
  v += from_lane<0x111, 0xf>(v); v += from_lane<0x112, 0xf>(v); v += from_lane<0x114, 0xf>(v); v += from_lane<0x118, 0xf>(v);
  v += from_lane<0x142, 0xa>(v); v += from_lane<0x143, 0xc>(v);
  return v;
}
template <int CTRL, int ROWS> __device__ __forceinline__ float from_lane(float v) { return __int_as_float(from_lane<CTRL, ROWS>(__float_as_int(v))); }
__device__ __forceinline__ float sum_of(float v) {
  v += from_lane<0x111, 0xf>(v); v += from_lane<0x112, 0xf>(v); v += from_lane<0x114, 0xf>(v); v += from_lane<0x118, 0xf>(v);
  v += from_lane<0x142, 0xa>(v); v += from_lane<0x143, 0xc>(v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float max_of_halves(float v) {  // of lanes i and i ^ 32
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float max_of_quarters(float v) {  // of lanes i, i ^ 16, i ^ 32, i ^ 48
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_of_halves(fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])));
}

// A row's maximum score and sum of weights if it sees nothing.  (A sum of zero alone can also mean that the scaled scores overflow, which gives NaN
// as the softmax of infinite scores does.)
__device__ __forceinline__ bool nothing_seen(float m, float l) { return m == -INFINITY && l == 0.f; }

// A sequence's part of the work: its tiles of R query rows, the positions that one of them can need at most, its chunks.
struct Share { int tiles, span, chunks, len; };
__device__ __forceinline__ Share share_of(const AttendArgs &a, const PagedSeq &s, int R) {
  Share x;
  x.tiles = (s.n * a.G + R - 1) / R;
  x.span = s.kv;
  if (a.window) x.span = (int)min((int64_t)s.kv, (int64_t)a.window + (R - 1) / a.G + 32);
  return x;
}
// `even`: the positions that every workgroup would have if the work could be cut anywhere.  A tile is cut into the number of equal chunks that
// comes nearest: so at most slots / 1.5 tiles are cut at all, into at most 4/3 slots chunks, and there are at most slots + tiles chunks.
__device__ __forceinline__ void cut(Share &x, int even, int align) {
  x.chunks = max(1, (x.span + even / 2) / even);
  x.len = ((x.span + x.chunks - 1) / x.chunks + align - 1) / align * align;
}
__device__ __forceinline__ int even_len(const AttendArgs &a, float work) {
  // the sum of up to 1024 roundings a lane (6e-5 of it): a little more keeps the bounds above
  const float even = work * a.one_slot * 1.0002f;
  return max(a.chunk_min, even < 1.e9f ? ((int)even + 128) & ~127 : 1 << 30);
}

// CUT false: unit `unit` of a pass's work, a chunk of a tile.  CUT true: the unit-th of the tiles that are cut.  part: the first of the
// tile's partial results (its chunks' lie `tiles` apart).  False: there is none.
template <bool CUT>
__device__ __forceinline__ bool find_work(const AttendArgs &a, int R, int align, int unit, Work &w) {
  const int lane = threadIdx.x & 63, B = a.p.B;
  auto lane_of = [](int v, int l) { return __builtin_amdgcn_readlane(v, l); };
  auto take = [&](int b, const PagedSeq &s, const Share &x, int u, int part) {
    w.b = b; w.s = s; w.chunks = x.chunks; w.chunk_len = x.len;
    // the last rows of a sequence see the most: their tiles start first
    w.tile = CUT ? u : x.tiles - 1 - u % x.tiles;
    w.chunk = CUT ? 0 : u / x.tiles;
    w.part = part + (CUT ? u : w.tile + w.chunk * x.tiles);
  };
  if (B <= 64) {
    PagedSeq s{0, 0, 0};
    int b = lane;
    if (lane < B) s = paged_seq(a.p, lane);
    Share x = share_of(a, s, R);
    if (B > 1) {  // longest first, which leaves the short ones to fill the end
      int rank = 0;
      for (int j = 0; j < B; ++j) {
        const int other = lane_of(x.span, j);
        rank += other > x.span || (other == x.span && j < lane);
      }
      if (lane >= B) rank = lane;
      s.row0 = __builtin_amdgcn_ds_permute(4 * rank, s.row0);
      s.n = __builtin_amdgcn_ds_permute(4 * rank, s.n);
      s.kv = __builtin_amdgcn_ds_permute(4 * rank, s.kv);
      b = __builtin_amdgcn_ds_permute(4 * rank, lane);
      x = share_of(a, s, R);
    }
    cut(x, even_len(a, sum_of((float)x.tiles * (float)x.span)), align);
    const int units = CUT ? (x.chunks > 1 ? x.tiles : 0) : x.tiles * x.chunks, to = sum_to(units);
    const int parts = x.chunks > 1 ? x.tiles * x.chunks : 0, parts_to = sum_to(parts);
    const unsigned long long here = __ballot(unit >= to - units && unit < to);
    if (!here) return false;
    const int l = __builtin_ctzll(here);
    take(lane_of(b, l), PagedSeq{lane_of(s.row0, l), lane_of(s.n, l), lane_of(s.kv, l)},
         Share{lane_of(x.tiles, l), 0, lane_of(x.chunks, l), lane_of(x.len, l)}, unit - lane_of(to - units, l), lane_of(parts_to - parts, l));
    return true;
  }
  const int per = (B + 63) / 64, first = lane * per, last = min(B, first + per);
  float work = 0.f;
  for (int b = first; b < last; ++b) {
    const Share x = share_of(a, paged_seq(a.p, b), R);
    work += (float)x.tiles * (float)x.span;
  }
  const int even = even_len(a, sum_of(work));
  int units = 0, parts = 0;
  for (int b = first; b < last; ++b) {
    Share x = share_of(a, paged_seq(a.p, b), R);
    cut(x, even, align);
    units += CUT ? (x.chunks > 1 ? x.tiles : 0) : x.tiles * x.chunks;
    parts += x.chunks > 1 ? x.tiles * x.chunks : 0;
  }
  const int to = sum_to(units), parts_to = sum_to(parts);
  const unsigned long long here = __ballot(unit >= to - units && unit < to);
  if (!here) return false;
  const int l = __builtin_ctzll(here);
  int at = lane_of(to - units, l), part = lane_of(parts_to - parts, l);
  for (int b = l * per; b < min(B, l * per + per); ++b) {
    const PagedSeq s = paged_seq(a.p, b);
    Share x = share_of(a, s, R);
    cut(x, even, align);
    const int n = CUT ? (x.chunks > 1 ? x.tiles : 0) : x.tiles * x.chunks;
    if (unit < at + n) {
      take(b, s, x, unit - at, part);
      return true;
    }
    at += n;
    part += x.chunks > 1 ? x.tiles * x.chunks : 0;
  }
  return false;
}
__device__ __forceinline__ Work in_scalars(const Work &w) {
  auto f = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  return Work{f(w.b), f(w.tile), f(w.chunk), f(w.chunks), f(w.chunk_len), f(w.part), PagedSeq{f(w.s.row0), f(w.s.n), f(w.s.kv)}};
}

// The positions [lo, hi) that any row of a tile sees, lo rounded down to a step.
__device__ __forceinline__ void tile_range(const AttendArgs &a, const PagedSeq &s, int tile, int R, int &lo, int &hi) {
  const int i0 = tile * R / a.G, i1 = min(s.n - 1, (tile * R + R - 1) / a.G), p0 = s.kv - s.n;
  hi = max(0, p0 + i1 + 1);
  lo = a.window ? max(0, p0 + i0 - a.window + 1) & ~31 : 0;
}

// ------------------------------------------------------------------ operands
template <class T> struct Mat;
template <> struct Mat<bf16_t> {
  static __device__ __forceinline__ f32x4_v run(u32x4_v a, u32x4_v b, f32x4_v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_v, a), __builtin_bit_cast(bf16x8_v, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {  // to nearest, one instruction
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_v){lo, hi}, bf16x2_v));
  }
};
template <> struct Mat<f16_t> {
  static __device__ __forceinline__ f32x4_v run(u32x4_v a, u32x4_v b, f32x4_v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_v, a), __builtin_bit_cast(f16x8_v, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_v){lo, hi}, f16x2_v));
  }
};
// log2 of the weight that the running maximum has.  fp16 has few small numbers: with the maximum's weight at 2^7 (2^15 where the maximum lags by 2^8), a weight
// is rounded by more than 2^-11 of itself only below 2^-21 of the row's largest, by 2^-32 of the largest then.  With the maximum's at 1
// 4000 positions of 2^-26 each counted for nothing.
template <class T> constexpr float top_weight() { return std::is_same<T, f16_t>::value ? 7.f : 0.f; }

// A lane's part of a step: its key rows of the two key tiles (KU units of 16 bytes each, units 4 kk + g), and 8 positions of
// VE = HD / 16 values, as loaded.
template <class T, class S, int HD> struct Step {
  static constexpr int E = 16 / sizeof(T), KU = HD / (4 * E), VE = HD / 16, VW = VE * sizeof(T) / 4;  // VW: words of a position's values
  u32x4_v k0[KU], k1[KU];
  uint32_t v[8][VW];
  // where the elements of a lane's kk-th operand of keys and queries begin
  static __device__ __forceinline__ int element(int kk, int g) { return (4 * kk + g) * E; }
};
// Of codes, a lane's units are the bytes 64 j + 16 g: two operands each.  With them come the scales of eight positions.
template <class T, int HD> struct Step<T, e4m3_t, HD> {
  static constexpr int E = 8, KU = HD / 32, VE = HD / 16, VW = VE / 2, RU = HD / 64, RW = VE / 4;
  u32x4_v k0[RU], k1[RU];
  uint32_t v[8][RW];
  uint2 ks, vs;
  static __device__ __forceinline__ int element(int kk, int g) { return 64 * (kk / 2) + 16 * g + 8 * (kk & 1); }
};
// byte i of eight, as a scale
__device__ __forceinline__ float scale_at(const uint2 &s, int i) { return scale_of((i < 4 ? s.x : s.y) >> (8 * (i & 3)) & 0xff); }

// (an absent page's loads are sent to page 0, which exists; what they bring is not used)
template <class T, class S, int HD>
__device__ __forceinline__ void load_keys(Step<T, S, HD> &f, const PagedArgs &p, size_t head_at, int hk, int page, int ks, int r, int g) {
  constexpr int UNITS = sizeof(f.k0) / 16;
  const unsigned char *kr = p.k + head_at + 16 * g + paged_row(p, page, ks + 8 * (r >> 2) + (r & 3));
  const size_t four = (size_t)p.pos_units << 6;
#pragma unroll
  for (int kk = 0; kk < UNITS; ++kk) {
    f.k0[kk] = *(const u32x4_v *)(kr + 64 * kk);
    f.k1[kk] = *(const u32x4_v *)(kr + four + 64 * kk);
  }
  if constexpr (std::is_same<S, e4m3_t>::value) f.ks = *(const uint2 *)(p.k_scale + paged_scale(p, page, hk, ks + 8 * (r >> 2)));
}
template <class T, class S, int HD>
__device__ __forceinline__ void load_values(Step<T, S, HD> &f, const PagedArgs &p, size_t head_at, int hk, int page, int ks, int r, int g) {
  constexpr int VB = sizeof(f.v) / 8;  // bytes of a position
  const unsigned char *vr = p.v + head_at + VB * r + paged_row(p, page, ks + 8 * g);
  const size_t one = (size_t)p.pos_units << 4;
#pragma unroll
  for (int i = 0; i < 8; ++i) __builtin_memcpy(f.v[i], __builtin_assume_aligned(vr + i * one, VB < 16 ? VB : 16), VB);
  if constexpr (std::is_same<S, e4m3_t>::value) f.vs = *(const uint2 *)(p.v_scale + paged_scale(p, page, hk, ks + 8 * g));
}

// S^T of a step: s0[i] <-> key 8g + i, s1[i] <-> key 8g + 4 + i of lane (query r, g)
template <class T, int KU>
__device__ __forceinline__ void scores(const u32x4_v (&k0)[KU], const u32x4_v (&k1)[KU], const u32x4_v (&q)[KU], float (&sv)[8]) {
  f32x4_v s0 = (f32x4_v){0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
  for (int kk = 0; kk < KU; ++kk) {
    if constexpr (sizeof(T) == 2) {
      s0 = Mat<T>::run(k0[kk], q[kk], s0);
      s1 = Mat<T>::run(k1[kk], q[kk], s1);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k0[kk][i]), __uint_as_float(q[kk][i]), s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k1[kk][i]), __uint_as_float(q[kk][i]), s1, 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { sv[i] = s0[i]; sv[4 + i] = s1[i]; }
}

// the 8 positions of element ht of a lane's values, as an operand
template <int VW>
__device__ __forceinline__ u32x4_v value_operand(const uint32_t (&v)[8][VW], int ht) {
  u32x4_v x;
#pragma unroll
  for (int d = 0; d < 4; ++d)
    x[d] = __builtin_amdgcn_perm(v[2 * d + 1][ht / 2], v[2 * d][ht / 2], (ht & 1) ? 0x07060302u : 0x05040100u);
  return x;
}

// Takes infinities and NaN out of a word of cached values; not zero if there were any.  (In integers: as conditions, a step's would fill the scalar
// registers.)
template <class T> __device__ __forceinline__ uint32_t drop_odd(uint32_t &w) {
  constexpr int top = sizeof(T) == 4 ? 31 : 15;  // of a value; two lie in a word of 16-bit ones
  constexpr uint32_t e = top == 31 ? 0x7f800000u : std::is_same<T, bf16_t>::value ? 0x7f807f80u : 0x7c007c00u, low = top == 31 ? 0x7fffffffu : 0x7fff7fffu;
  const uint32_t finite = (((w & e) ^ e) + low) & ~low;  // a value's top bit, where its exponent is not all ones
  const uint32_t keep = (finite - (finite >> top)) | finite;
  w &= keep;
  return ~keep;
}
// The value if it is infinite or NaN, else zero.
template <class T> __device__ __forceinline__ float only_odd(T t) {
  if constexpr (std::is_same<T, e4m3_t>::value) {
    return (t.v & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f;
  } else {
    const float v = Conv<T>::ld(&t, 0);
    return fabsf(v) < INFINITY ? 0.f : v;
  }
}

// Which unit of work and key head a workgroup takes.  A position's heads lie side by side, as do their scales: with 8 bits a head has a line of memory
// or a part of one.  So eight heads of one unit run on one XCD (workgroups are dealt to the eight in turn), and lines that they share come there once:
// 64 sequences x 4 rows of 32 heads of 128 78.5 -> 74.4 us, of 64 heads of 64 113 -> 88.  (Grids are whole groups of 64; units behind the last have no work.)
template <bool C8> __device__ __forceinline__ void my_unit(int Hk, int &unit, int &hk) {
  const int i = blockIdx.x;
  if (C8 && Hk % 8 == 0) {
    const int eight = i / 64 * 8 + i % 8;  // of eight heads
    unit = eight / (Hk / 8);
    hk = eight % (Hk / 8) * 8 + i / 8 % 8;
  } else {
    unit = i / Hk;
    hk = i % Hk;
  }
}

// ------------------------------------------------------------------ few query rows a tile: the waves share the positions
// Workgroups that a CU holds at a time: by registers, which its launch bound holds the compiler to.
constexpr int attend_resident(int dtype_bytes, int HD, int QT) {
  if (dtype_bytes == 4) return HD == 64 && QT == 1 ? 3 : HD == 64 ? 2 : 1;
  return QT == 1 ? (HD == 64 ? 4 : 3) : QT == 2 ? (HD == 64 ? 3 : 1) : QT == 4 ? 1 : QT == 8 ? 2 : 1;
}
template <class T, class S, int HD, int QT>
__global__ __launch_bounds__(256, attend_resident(sizeof(T), HD, QT)) void k_paged_attend(AttendArgs a) {
  typedef Step<T, S, HD> St;
  constexpr bool C8 = std::is_same<S, e4m3_t>::value;
  constexpr int R = 16 * QT, HT = HD / 16, KU = St::KU, VE = St::VE, LD = HD + 4;
  __shared__ float sh_o[PA_WAVES][16][LD];
  __shared__ float sh_m[PA_WAVES][R], sh_l[PA_WAVES][R];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int Hk = a.p.n_kv_heads;
  int unit, hk;
  my_unit<C8>(Hk, unit, hk);
  Work w;
  if (!find_work<false>(a, R, 128, unit, w)) return;
  w = in_scalars(w);
  const PagedSeq s = w.s;
  int lo, hi;
  tile_range(a, s, w.tile, R, lo, hi);
  const int k_begin = lo + w.chunk * w.chunk_len, k_end = hi - k_begin > w.chunk_len ? k_begin + w.chunk_len : hi;
  const bool several = w.chunks > 1;

  // this lane's query rows: tile row 16 t + r
  int pos[QT];
  u32x4_v q[QT][KU];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int f = w.tile * R + 16 * t + r, i = f / a.G;
    const bool on = f < s.n * a.G;
    pos[t] = on ? s.kv - s.n + i : -1;
    const T *src = (const T *)a.q + (on ? (s.row0 + i) * a.q_stride + (hk * a.G + f - i * a.G) * HD : 0);
#pragma unroll
    for (int kk = 0; kk < KU; ++kk) q[t][kk] = on ? *(const u32x4_v *)(src + St::element(kk, g)) : (u32x4_v){0, 0, 0, 0};
  }
  // every row of the tile sees all positions [see_lo, see_hi)
  const int i0 = w.tile * R / a.G, i1 = min(s.n - 1, (w.tile * R + R - 1) / a.G);
  const int see_hi = s.kv - s.n + i0 + 1, see_lo = a.window ? s.kv - s.n + i1 - a.window + 1 : 0;
  // the first position that any of them sees (the first step, a multiple of 32, can begin before it)
  const int any_lo = a.window ? s.kv - s.n + i0 - a.window + 1 : 0;

  auto all_see = [&](int ks) { return ks >= see_lo && ks + 32 <= min(see_hi, k_end); };

  float m[QT], l[QT];
  f32x4_v acc[QT][HT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) acc[t][ht] = (f32x4_v){0.f, 0.f, 0.f, 0.f};
  }

  const size_t head_at = (size_t)hk * a.p.head_units << 4;  // bytes
  // Pages are looked up two steps ahead, of positions behind the end the last one's.  They are checked where they are used: a check here would wait
  // for the load, and with it for every load before it.
  const int ks0 = k_begin + 32 * wv;
  const int32_t *table = a.p.pages + w.b * a.p.pages_stride;
  auto page_at = [&](int pos) { return table[(unsigned)min(pos, k_end - 1) >> a.p.page_shift]; };
  auto is_there = [&](int page) { return (unsigned)page < (unsigned)a.p.n_pages; };
  St f;
  int pv = -1, pk_next = -1, pv_next = -1;
  if (ks0 < k_end) {
    const int pk = page_at(ks0 + 8 * (r >> 2));
    pv = page_at(ks0 + 8 * g);
    load_keys<T, S, HD>(f, a.p, head_at, hk, is_there(pk) ? pk : 0, ks0, r, g);
    load_values<T, S, HD>(f, a.p, head_at, hk, is_there(pv) ? pv : 0, ks0, r, g);
    pk_next = page_at(ks0 + 128 + 8 * (r >> 2));
    pv_next = page_at(ks0 + 128 + 8 * g);
  }
  uint32_t odd = 0;
  // (the last step is a copy without loads: loads behind a branch would make the waits in front of the products wait for all of them)
  auto step = [&](int ks, auto more_) {
    constexpr bool more = decltype(more_)::value;
    const int pk = pk_next, pv_then = pv_next;
    if constexpr (more) {
      pk_next = page_at(ks + 256 + 8 * (r >> 2));
      pv_next = page_at(ks + 256 + 8 * g);
    }
    float p[QT][8];
    if constexpr (C8) {
      const float s0 = scale_of(f.ks.x >> (8 * (r & 3)) & 0xff), s1 = scale_of(f.ks.y >> (8 * (r & 3)) & 0xff);
      u32x4_v k0[KU], k1[KU];
#pragma unroll
      for (int j = 0; j < KU / 2; ++j) {
        decode16<T>(f.k0[j], s0, k0[2 * j], k0[2 * j + 1]);
        decode16<T>(f.k1[j], s1, k1[2 * j], k1[2 * j + 1]);
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) scores<T, KU>(k0, k1, q[t], p[t]);
    } else {
#pragma unroll
      for (int t = 0; t < QT; ++t) scores<T, KU>(f.k0, f.k1, q[t], p[t]);
    }
    // the keys are used: the next step's take their registers while the weights are worked out, and the next values' these values'
    if constexpr (more) load_keys<T, S, HD>(f, a.p, head_at, hk, is_there(pk) ? pk : 0, ks + 128, r, g);
    // keys of this lane's scores: ks + 8g + i, in page pv
    const bool there = is_there(pv), alike = all_see(ks), whole = alike && __all(there);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float(&sv)[8] = p[t];
      if (!whole) {
        const int from = a.window ? pos[t] - a.window + 1 : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = ks + 8 * g + i;
          sv[i] = there && key <= pos[t] && key >= from && key < k_end ? sv[i] : -INFINITY;
        }
      }
      const float top = max_of_quarters(fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7]))));
      if (__any(top > m[t])) {
        const float mn = fmaxf(m[t], top);
        const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[t] - mn) * a.sl2);
        m[t] = mn;
        l[t] *= corr;
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) { acc[t][ht][0] *= corr; acc[t][ht][1] *= corr; acc[t][ht][2] *= corr; acc[t][ht][3] *= corr; }
      }
      const float off = m[t] == -INFINITY ? 0.f : fmaf(m[t], a.sl2, -top_weight<T>());
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sv[i] = __builtin_amdgcn_exp2f(fmaf(sv[i], a.sl2, -off));
        l[t] += sv[i];
      }
    }
    uint32_t expanded[C8 ? 8 : 1][St::VW];
    if constexpr (C8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float scale = scale_at(f.vs, i);
#pragma unroll
        for (int x = 0; x < St::RW; ++x) {
          expanded[i][2 * x] = decode2<T, false>(f.v[i][x], scale);
          expanded[i][2 * x + 1] = decode2<T, true>(f.v[i][x], scale);
        }
      }
    }
    uint32_t(&v)[8][St::VW] = [&]() -> auto & { if constexpr (C8) return expanded; else return f.v; }();
    if (!whole) {  // positions that no row of the tile sees: their values, whatever they are, become zeros
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = ks + 8 * g + i;
        const bool live = there && key >= any_lo && key < k_end;
#pragma unroll
        for (int x = 0; x < St::VW; ++x) v[i][x] = live ? v[i][x] : 0u;
      }
      // Positions that some of the tile's rows see and others do not: a weight of zero does not keep an infinity or a NaN out of a
      // product, so such values leave here and are added at the end for the rows that see them.
      if (i0 != i1 && !alike) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int x = 0; x < St::VW; ++x) odd |= drop_odd<T>(v[i][x]);
      }
    }
    u32x4_v y[QT];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int d = 0; d < 4; ++d) y[t][d] = Mat<T>::pack2(p[t][2 * d], p[t][2 * d + 1]);
    }
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) {
      if constexpr (sizeof(T) == 2) {
        const u32x4_v x = value_operand(v, ht);
#pragma unroll
        for (int t = 0; t < QT; ++t) acc[t][ht] = Mat<T>::run(x, y[t], acc[t][ht]);
      } else {
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            acc[t][ht] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][ht]), p[t][i], acc[t][ht], 0, 0, 0);
      }
    }
    if constexpr (more) load_values<T, S, HD>(f, a.p, head_at, hk, is_there(pv_then) ? pv_then : 0, ks + 128, r, g);
    pv = pv_then;
  };
  if (ks0 < k_end) {
    int ks = ks0;
    for (; ks + 128 < k_end; ks += 128) step(ks, std::true_type());
    step(ks, std::false_type());
  }

  if (__any(odd != 0)) {  // this wave's steps that hold positions outside [see_lo, see_hi) again
    for (int ks = ks0; ks < k_end; ks += 128) {
      if (all_see(ks)) continue;
      for (int key = ks; key < min(ks + 32, k_end); ++key) {
        const int page = paged_page(a.p, w.b, key);
        if (page < 0) continue;
        const S *src = (const S *)(a.p.v + head_at + paged_row(a.p, page, key)) + 4 * VE * g;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[VE];
#pragma unroll
          for (int ht = 0; ht < HT; ++ht) v[ht] = only_odd<S>(src[VE * e + ht]);
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            const bool sees = key <= pos[t] && !(a.window && key <= pos[t] - a.window);
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) acc[t][ht][e] += sees ? v[ht] : 0.f;
          }
          __builtin_amdgcn_sched_barrier(0);  // (or all their conditions are held at once)
        }
      }
    }
  }

  // the waves' maxima and sums, then their outputs, 16 query rows at a time
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
    if (g == 0) { sh_m[wv][16 * t + r] = m[t]; sh_l[wv][16 * t + r] = l[t]; }
  }
  __syncthreads();
  const int64_t slot = ((int64_t)w.part * Hk + hk) * R;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float mt = -INFINITY;
#pragma unroll
    for (int x = 0; x < PA_WAVES; ++x) mt = fmaxf(mt, sh_m[x][16 * t + r]);
    const float c = m[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[t] - mt) * a.sl2);
    if (t) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int ht = 0; ht < HT; ++ht) sh_o[wv][r][VE * (4 * g + e) + ht] = acc[t][ht][e] * c;
    __syncthreads();
    // thread: query row tid / 16, VE elements from VE * (tid % 16) on
    const int row = threadIdx.x >> 4, d0 = VE * (threadIdx.x & 15), f = w.tile * R + 16 * t + row;
    if (f < s.n * a.G) {
      float mr = -INFINITY, lr = 0.f, o[VE];
#pragma unroll
      for (int x = 0; x < PA_WAVES; ++x) mr = fmaxf(mr, sh_m[x][16 * t + row]);
#pragma unroll
      for (int x = 0; x < PA_WAVES; ++x)
        lr += sh_l[x][16 * t + row] * (sh_m[x][16 * t + row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((sh_m[x][16 * t + row] - mr) * a.sl2));
#pragma unroll
      for (int d = 0; d < VE; ++d) o[d] = ((sh_o[0][row][d0 + d] + sh_o[1][row][d0 + d]) + sh_o[2][row][d0 + d]) + sh_o[3][row][d0 + d];
      if (several) {
        float *dst = a.part + (slot + 16 * t + row) * HD + d0;
#pragma unroll
        for (int d = 0; d < VE; ++d) dst[d] = o[d];
        if (d0 == 0) { a.ml[(slot + 16 * t + row) * 2] = mr; a.ml[(slot + 16 * t + row) * 2 + 1] = lr; }
      } else {
        const bool none = nothing_seen(mr, lr);
        const float inv = 1.f / lr;
        const int i = f / a.G;
        T *dst = (T *)a.out + (s.row0 + i) * a.out_stride + (hk * a.G + f - i * a.G) * HD + d0;
#pragma unroll
        for (int d = 0; d < VE; ++d) Conv<T>::st(dst, d, none ? 0.f : o[d] * inv);
      }
    }
  }
}

// ------------------------------------------------------------------ many query rows: the waves share the cached rows through LDS
typedef __attribute__((ext_vector_type(16))) float f32x16_v;
template <class T> __device__ __forceinline__ f32x16_v mat32(u32x4_v a, u32x4_v b, f32x16_v c) {
  if constexpr (std::is_same<T, bf16_t>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_v, a), __builtin_bit_cast(bf16x8_v, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_v, a), __builtin_bit_cast(f16x8_v, b), c, 0, 0, 0);
}
// 16 bytes a lane from its own address to LDS byte `lds` + 16 lane
__device__ __forceinline__ void lanes_to_lds(const void *p, unsigned lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds), "v"(p) : "memory");
}
// The largest of top and x[0 .. 13].  Written as fmaxf, every score is first brought to canonical form by an instruction of its own.  The compiler
// does not see what asm reads: top has to come from an instruction that reads the products' last result, so that it waits for them.
__device__ __forceinline__ float max14(float top, const f32x16_v &x) {
  asm("v_max3_f32 %0, %0, %1, %2\n\tv_max3_f32 %0, %0, %3, %4\n\tv_max3_f32 %0, %0, %5, %6\n\tv_max3_f32 %0, %0, %7, %8\n\t"
      "v_max3_f32 %0, %0, %9, %10\n\tv_max3_f32 %0, %0, %11, %12\n\tv_max3_f32 %0, %0, %13, %14"
      : "+v"(top)
      : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]), "v"(x[8]), "v"(x[9]), "v"(x[10]), "v"(x[11]),
        "v"(x[12]), "v"(x[13]));
  return top;
}

// A workgroup of NW waves takes 32 NW query rows, 32 a wave, and walks the positions in tiles of KT = 16 NW (heads of 128) or 32 NW (of 64):
// 4 NW KB of keys and as much of values, in LDS in operand order, twice.  32x32x16 products: a lane owns one query (lane % 32) and half of
// every 16 keys, so a row's maximum takes one exchange.  Keys go straight to LDS, [key][unit of 16 bytes], a row's units exchanged by its number so
// that reading one unit of 32 rows meets every bank; of values a thread loads 8 positions of 4 elements and turns them round on
// the way to LDS.  The maximum follows the scores only when they have grown
// by 2^8: weights up to 2^8 are as exact in 16 bits as weights up to 1 (fp16: up to 2^15 as those up to 2^7), the sums are fp32, and most tiles
// then rescale nothing.
// Chunks of up to 2048 rows over 8192 positions, 32 heads over 8, bf16: 417 us (913 TFLOP/s), products busy 42 % of the clocks.  Of codes: 414 us; their
// decoding, once for all rows of the workgroup, runs beside the products.
constexpr int VALU = 0x2, MATRIX = 0x8, DS_READ = 0x100;  // kinds of instructions that sched_group_barrier tells apart
constexpr int pc_lds(int NW) { return 4 * NW * 256 * 16; }

template <class T, class S, int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_paged_chunk(AttendArgs a) {
  constexpr bool C8 = std::is_same<S, e4m3_t>::value;
  constexpr int R = 32 * NW, NC = HD / 8, KK = HD / 16, DT = HD / 32, KT = 256 * NW / NC, VC = HD / 4, IPT = 32 / VC, UNITS = KT * NC;
  extern __shared__ __attribute__((aligned(16))) u32x4_v pc_smem[];  // [2] keys [KT][NC], [2] values [KT / 16][DT][2][32]
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const int Hk = a.p.n_kv_heads, unit = blockIdx.x / Hk, hk = blockIdx.x % Hk;
  Work w;
  if (!find_work<false>(a, R, KT, unit, w)) return;
  w = in_scalars(w);
  const PagedSeq s = w.s;
  int lo, hi;
  tile_range(a, s, w.tile, R, lo, hi);
  const int k_begin = lo + w.chunk * w.chunk_len, k_end = hi - k_begin > w.chunk_len ? k_begin + w.chunk_len : hi;
  const int rows = s.n * a.G, p0 = s.kv - s.n;

  // this lane's query, and what the wave's queries see: all of them [see_lo, see_hi), any of them [any_lo, any_hi)
  const int f0 = w.tile * R + 32 * wv, f = f0 + col, qi = f / a.G;
  const bool on = f < rows;
  const int pos = on ? p0 + qi : -1;
  const int first = p0 + f0 / a.G, last = p0 + min(f0 + 31, rows - 1) / a.G;
  const int see_hi = first + 1, see_lo = a.window ? last - a.window + 1 : 0, any_hi = f0 < rows ? last + 1 : 0, any_lo = a.window ? first - a.window + 1 : 0;
  u32x4_v q[KK];
  {
    const T *src = (const T *)a.q + (on ? (s.row0 + qi) * a.q_stride + (hk * a.G + f - qi * a.G) * HD : 0) + 8 * h;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = on ? *(const u32x4_v *)(src + 16 * kk) : (u32x4_v){0, 0, 0, 0};
  }

  // staging
  const int vc = threadIdx.x % VC, kg = threadIdx.x / VC;
  const size_t head_at = (size_t)hk * a.p.head_units << 4;  // bytes
  const unsigned char *k_base = a.p.k + head_at, *v_base = a.p.v + head_at + 4 * sizeof(S) * vc;
  const int32_t *table = a.p.pages + w.b * a.p.pages_stride;
  const size_t pos_bytes = (size_t)a.p.pos_units << 4;
  // Pages are looked up a tile ahead, of positions behind the end the last one's.  They are checked where they are used: a check here would wait
  // for the load, and with it for every load before it.
  auto page_at = [&](int pos) { return table[(unsigned)min(pos, k_end - 1) >> a.p.page_shift]; };
  auto is_there = [&](int page) { return (unsigned)page < (unsigned)a.p.n_pages; };
  auto row_at = [&](int page, int pos) { return paged_row(a.p, is_there(page) ? page : 0, pos); };
  // Row 32 u + 16 x + 8 y + 4 z + e of a key tile holds key 32 u + 16 x + 8 z + 4 y + e.  Wave instruction `it` fills 64 / NC rows; its
  // lanes' keys lie in one of two groups of eight positions, kgrp[it's].
  const int kgrp0 = NC == 16 ? 2 * wv : 4 * wv + (lane >> 5), kgrp1 = kgrp0 + (NC == 16 ? 1 : 2);
  const int krow = NC == 16 ? 16 * wv + (lane >> 4) : 32 * wv + 8 * (lane >> 5) + (lane >> 3 & 3);  // key of it = 0
  uint32_t x[8][2];
  int x_page;
  // Codes come through registers: a thread's are the unit kc of the keys ck and ck + KT / 2, and four elements of eight values.
  constexpr int RC = HD / 16;
  const int kc = threadIdx.x % RC, ck = threadIdx.x / RC;
  u32x4_v raw_k[C8 ? 2 : 1];
  uint32_t raw_ks[2], raw_v[C8 ? 8 : 1];
  uint2 raw_vs;
  struct Pages { int k[2], v; };
  auto pages_of = [&](int ks) {
    if constexpr (C8) return Pages{{page_at(ks + ck), page_at(ks + KT / 2 + ck)}, page_at(ks + 8 * kg)};
    else return Pages{{page_at(ks + 8 * kgrp0), page_at(ks + 8 * kgrp1)}, page_at(ks + 8 * kg)};
  };
  auto fetch = [&](int ks, const Pages &pg, int kbuf) {
    if constexpr (C8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int pos = ks + KT / 2 * i + ck, page = is_there(pg.k[i]) ? pg.k[i] : 0;
        raw_k[i] = *(const u32x4_v *)(k_base + paged_row(a.p, page, pos) + 16 * kc);
        raw_ks[i] = a.p.k_scale[paged_scale(a.p, page, hk, pos)];
      }
      const int page = is_there(pg.v) ? pg.v : 0;
      const unsigned char *src = v_base + paged_row(a.p, page, ks + 8 * kg);
      x_page = pg.v;
#pragma unroll
      for (int i = 0; i < 8; ++i) raw_v[i] = *(const uint32_t *)(src + i * pos_bytes);
      raw_vs = *(const uint2 *)(a.p.v_scale + paged_scale(a.p, page, hk, ks + 8 * kg));
      return;
    }
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int key = krow + (NC == 16 ? 8 * (it & 1) + 4 * (it >> 1) : 16 * (it >> 1) + 4 * (it & 1));
      const int unit = NC == 16 ? (lane ^ (lane >> 4)) % 16 ^ 4 * it : (lane ^ (lane >> 3)) % 8;  // by the row's number
      const unsigned char *src = k_base + row_at(pg.k[NC == 16 ? it & 1 : it >> 1], ks + key) + 16 * unit;
      lanes_to_lds(src, (unsigned)((kbuf * UNITS + (wv * 4 + it) * 64) * 16));
    }
    const unsigned char *src = v_base + row_at(pg.v, ks + 8 * kg);
    x_page = pg.v;
#pragma unroll
    for (int i = 0; i < 8; ++i) __builtin_memcpy(x[i], __builtin_assume_aligned(src + i * pos_bytes, 8), 8);
  };
  // All rows of the workgroup see [all_lo, all_hi).  Beyond, where some do and others do not, a weight of zero does not keep an infinity or a NaN
  // out of a product: from tiles of positions that reach beyond (odd_tile) all such values leave here, and are added at the end for
  // the rows that see them.
  const int all_hi = p0 + w.tile * R / a.G + 1, all_lo = a.window ? p0 + min(w.tile * R + R - 1, rows - 1) / a.G - a.window + 1 : 0;
  auto odd_tile = [&](int ks) { return ks + KT > all_hi || ks < all_lo; };
  uint32_t odd = 0;
  auto store = [&](int ks, int vbuf) {
    if constexpr (C8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int key = KT / 2 * i + ck, row = (key & ~12) | (key & 4) << 1 | (key & 8) >> 1;
        u32x4_v y0, y1, *kb = pc_smem + vbuf * UNITS + row * NC;
        decode16<T>(raw_k[i], scale_of(raw_ks[i]), y0, y1);
        kb[(2 * kc) ^ (row & (NC - 1))] = y0;
        kb[(2 * kc + 1) ^ (row & (NC - 1))] = y1;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float scale = scale_at(raw_vs, i);
        x[i][0] = decode2<T, false>(raw_v[i], scale);
        x[i][1] = decode2<T, true>(raw_v[i], scale);
      }
    }
    const int live = is_there(x_page) ? k_end - (ks + 8 * kg) : 0;  // positions behind the end hold anything
    if (live < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i][0] = i < live ? x[i][0] : 0u; x[i][1] = i < live ? x[i][1] : 0u; }
    }
    if (odd_tile(ks)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) { odd |= drop_odd<T>(x[i][0]); odd |= drop_odd<T>(x[i][1]); }
    }
    u32x4_v *vb = pc_smem + (2 + vbuf) * UNITS + (kg >> 1) * DT * 64 + (kg & 1) * 32 + vc;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4_v y;
#pragma unroll
      for (int d = 0; d < 4; ++d) y[d] = __builtin_amdgcn_perm(x[2 * d + 1][i / 2], x[2 * d][i / 2], (i & 1) ? 0x07060302u : 0x05040100u);
      vb[(i / IPT) * 64 + VC * (i % IPT)] = y;
    }
  };
  // loads to LDS have landed, reads of LDS are done; behind the barrier everyone's
  auto meet = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0), known to the compiler
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  float m = -INFINITY, l = 0.f;
  const float grow = fminf(8.f / a.sl2, 3.4e38f);  // (finite: the maximum starts at -infinity)
  f32x16_v acc[DT];
#pragma unroll
  for (int j = 0; j < DT; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;

  // score e of sc[u]: key ks + 32 u + 16 (e / 8) + 8 h + e % 8
  f32x16_v sc[2];
  // The two tiles' chains of products in turn, so that a product need not wait for the one issued before it (430 -> 421 us for chunks of up to
  // 2048 rows).
  auto key_products = [&](const u32x4_v *kb) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int u = 0; u < 2; ++u) sc[u] = mat32<T>(kb[(32 * u + col) * NC + ((2 * kk + h) ^ (col & (NC - 1)))], q[kk], sc[u]);
    // four reads ahead of the products (left to itself the compiler has one or two: 443 -> 432 us for chunks of up to 2048 rows)
    __builtin_amdgcn_sched_group_barrier(DS_READ, 4, 0);
#pragma unroll
    for (int i = 0; i < 2 * KK - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(MATRIX, 1, 0);
      __builtin_amdgcn_sched_group_barrier(DS_READ, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(MATRIX, 4, 0);
  };
  // the maximum follows where it has to; -> what is taken off the scaled scores
  auto follow = [&]() {
    const float last2 = fmaxf(fmaxf(sc[0][14], sc[0][15]), fmaxf(sc[1][14], sc[1][15]));
    const float top = max_of_halves(max14(max14(last2, sc[0]), sc[1]));
    if (__any(top > m + grow)) {
      const float mn = fmaxf(m, top), corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.sl2);
      m = mn;
      l *= corr;
#pragma unroll
      for (int j = 0; j < DT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][e] *= corr;
    }
    return m == -INFINITY ? 0.f : fmaf(m, a.sl2, -top_weight<T>());
  };
  auto weights = [&](int y, float off) {  // of the 16 keys y of a step
    u32x4_v p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[y / 2][8 * (y & 1) + 2 * i], a.sl2, -off));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[y / 2][8 * (y & 1) + 2 * i + 1], a.sl2, -off));
      l += p0 + p1;
      p[i] = Mat<T>::pack2(p0, p1);
    }
    return p;
  };
  // Tile t lies in buffers t % 2.  Lane i of a wave also looks whether the i-th eight positions of a tile are there at all.
  auto there_at = [&](int ks) { return page_at(ks + 8 * (lane % (KT / 8))); };
  unsigned present = 0;
  Pages pages{{-1, -1}, -1};
  if (k_begin < k_end) {
    const int there = there_at(k_begin);
    fetch(k_begin, pages_of(k_begin), 0);
    pages = pages_of(k_begin + KT);
    store(k_begin, 0);
    present = (unsigned)__ballot(is_there(there));
  }
  meet();
  int buf = 0;
  for (int ks0 = k_begin; ks0 < k_end; ks0 += KT, buf ^= 1) {
    // The next tile's loads land while this one is worked on.  Behind the last tile they bring rows of the last position's page (page 0's if it
    // is absent), which nothing reads: no branch keeps the address arithmetic from the products' shadow.
    fetch(ks0 + KT, pages, buf ^ 1);
    pages = pages_of(ks0 + 2 * KT);
    const int there = there_at(ks0 + KT);
    const u32x4_v *kb = pc_smem + buf * UNITS, *vb = pc_smem + (2 + buf) * UNITS + h * 32 + col;
#pragma unroll
    for (int step = 0; step < KT / 64; ++step) {
      const int ks = ks0 + 64 * step;
      const unsigned here = present >> (8 * step) & 0xff;
      const u32x4_v *ksrc = kb + 64 * step * NC, *vs = vb + step * 4 * DT * 64;
      if (ks >= any_hi || ks + 64 <= any_lo || ks >= k_end) continue;
      key_products(ksrc);
      if (ks < see_lo || ks + 64 > min(see_hi, k_end) || here != 0xff) {
        const int from = a.window ? pos - a.window + 1 : 0;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int group = 4 * u + 2 * (e >> 3) + h, key = ks + 8 * group + (e & 7);
            sc[u][e] = key <= pos && key >= from && key < k_end && (here >> group & 1) ? sc[u][e] : -INFINITY;
          }
      }
      __builtin_amdgcn_s_setprio(1);  // over the other wave's products, which run on by themselves (419 -> 413 us)
      const float off = follow();
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const u32x4_v p = weights(y, off);
#pragma unroll
        for (int j = 0; j < DT; ++j) acc[j] = mat32<T>(vs[(y * DT + j) * 64], p, acc[j]);
      }
      // the later keys' weights between the earlier keys' products
      __builtin_amdgcn_sched_group_barrier(DS_READ, 4, 0);
      __builtin_amdgcn_sched_group_barrier(VALU, 30, 0);
#pragma unroll
      for (int i = 0; i < 4 * DT - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(MATRIX, 1, 0);
        __builtin_amdgcn_sched_group_barrier(DS_READ, 1, 0);
        __builtin_amdgcn_sched_group_barrier(VALU, 28 / DT, 0);
      }
      __builtin_amdgcn_sched_group_barrier(MATRIX, 4, 0);
      __builtin_amdgcn_s_setprio(0);
    }
    store(ks0 + KT, buf ^ 1);
    present = (unsigned)__ballot(is_there(there));
    meet();
  }

  l += __shfl_xor(l, 32, 64);
  uint32_t *flags = (uint32_t *)pc_smem;  // nothing reads the tiles any more
  if (lane == 0) flags[wv] = 0;
  if (odd) flags[wv] = 1;
  meet();
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) any |= flags[i];
  if (any) {
    const int from = a.window ? pos - a.window + 1 : 0;
    for (int key = k_begin; key < k_end; ++key) {
      if ((key - k_begin) % KT == 0 && !odd_tile(key)) { key += KT - 1; continue; }
      const int page = page_at(key);
      if (!is_there(page) || key > pos || key < from) continue;
      const S *src = (const S *)(a.p.v + head_at + paged_row(a.p, page, key));
#pragma unroll
      for (int j = 0; j < DT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int row = 8 * (e >> 2) + 4 * h + (e & 3);
          acc[j][e] += only_odd<S>(src[4 * (row % VC) + j * IPT + row / VC]);
        }
    }
  }
  if (!on) return;
  // element 4 c + i of the query lies in tile i / IPT, row c + VC (i % IPT); a lane holds the rows 8 (e / 4) + 4 h + e % 4
  const bool several = w.chunks > 1;
  const int64_t at = ((int64_t)w.part * Hk + hk) * R + 32 * wv + col;
  const bool none = nothing_seen(m, l);
  const float inv = 1.f / l;
  T *dst = (T *)a.out + (s.row0 + qi) * a.out_stride + (hk * a.G + f - qi * a.G) * HD;
  if (several && h == 0) { a.ml[at * 2] = m; a.ml[at * 2 + 1] = l; }
#pragma unroll
  for (int x = 0; x < VC / 8; ++x) {  // rows 8 x + 4 h + y: 16 elements in a row
    const int d = 4 * (8 * x + 4 * h);
    float o[16];
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[4 * y + i] = acc[i / IPT][4 * (x + VC / 8 * (i % IPT)) + y];
    if (several) {
#pragma unroll
      for (int y = 0; y < 4; ++y) *(f32x4_v *)(a.part + at * HD + d + 4 * y) = (f32x4_v){o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]};
    } else {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        u32x4_v v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = Mat<T>::pack2(none ? 0.f : o[8 * y + 2 * i] * inv, none ? 0.f : o[8 * y + 2 * i + 1] * inv);
        *(u32x4_v *)(dst + d + 8 * y) = v;
      }
    }
  }
}

// Joins the chunks of the tiles that are cut: a workgroup takes 16 query rows of one, a thread VE elements of a row.
template <class T, int HD, int QT>
__global__ __launch_bounds__(256) void k_paged_join(AttendArgs a, int align) {
  constexpr int R = 16 * QT, VE = HD / 16, AHEAD = 8;
  const int Hk = a.p.n_kv_heads, t = blockIdx.x % QT, unit = blockIdx.x / QT / Hk, hk = blockIdx.x / QT % Hk;
  Work w;
  if (!find_work<true>(a, R, align, unit, w)) return;
  w = in_scalars(w);
  const PagedSeq s = w.s;
  const int row = threadIdx.x >> 4, d0 = VE * (threadIdx.x & 15), f = w.tile * R + 16 * t + row;
  if (f >= s.n * a.G) return;
  const int64_t next = (int64_t)((s.n * a.G + R - 1) / R) * Hk * R, at = ((int64_t)w.part * Hk + hk) * R + 16 * t + row;
  const float2 *ml = (const float2 *)a.ml + at;
  const float *part = a.part + at * HD + d0;
  float m = -INFINITY, l = 0.f, o[VE];
  for (int c0 = 0; c0 < w.chunks; c0 += AHEAD) {
    float mc[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) mc[i] = ml[min(c0 + i, w.chunks - 1) * next].x;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) m = fmaxf(m, mc[i]);
  }
#pragma unroll
  for (int d = 0; d < VE; ++d) o[d] = 0.f;
  for (int c0 = 0; c0 < w.chunks; c0 += AHEAD) {
    float2 x[AHEAD];
    f32x4_v y[AHEAD][VE / 4];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t c = min(c0 + i, w.chunks - 1) * next;
      x[i] = ml[c];
#pragma unroll
      for (int d = 0; d < VE / 4; ++d) y[i][d] = *(const f32x4_v *)(part + c * HD + 4 * d);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (c0 + i >= w.chunks) break;
      const float wt = x[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[i].x - m) * a.sl2);
      l += x[i].y * wt;
#pragma unroll
      for (int d = 0; d < VE; ++d) o[d] += y[i][d / 4][d % 4] * wt;
    }
  }
  const bool none = nothing_seen(m, l);
  const float inv = 1.f / l;
  const int i = f / a.G;
  T *dst = (T *)a.out + (s.row0 + i) * a.out_stride + (hk * a.G + f - i * a.G) * HD + d0;
#pragma unroll
  for (int d = 0; d < VE; ++d) Conv<T>::st(dst, d, none ? 0.f : o[d] * inv);
}

// The same with a wave a query row: a lane a chunk for maxima and sums, then a quarter every fourth chunk for the elements.  For a few rows that are cut
// into many chunks, which 16 lanes join one after the other: one row of 32 heads over 8, fp16, 32000 positions in 63 chunks of 8 bits, the call 38.1 us
// with 16 lanes a row, 24.7 with running maxima in every quarter, 21.2 so.
template <class T, int HD, int QT>
__global__ __launch_bounds__(256) void k_paged_join_rows(AttendArgs a, int align) {
  constexpr int R = 16 * QT, VE = HD / 16, AHEAD = 8;
  const int Hk = a.p.n_kv_heads, unit = blockIdx.x / (R / 4) / Hk, hk = blockIdx.x / (R / 4) % Hk;
  Work w;
  if (!find_work<true>(a, R, align, unit, w)) return;
  w = in_scalars(w);
  const PagedSeq s = w.s;
  const int lane = threadIdx.x & 63, row = blockIdx.x % (R / 4) * 4 + (threadIdx.x >> 6), quarter = lane >> 4, d0 = VE * (lane & 15), f = w.tile * R + row;
  if (f >= s.n * a.G) return;
  const int64_t next = (int64_t)((s.n * a.G + R - 1) / R) * Hk * R, at = ((int64_t)w.part * Hk + hk) * R + row;
  const float2 *ml = (const float2 *)a.ml + at;
  const float *part = a.part + at * HD + d0;
  float m = -INFINITY, l = 0.f, o[VE];
#pragma unroll
  for (int d = 0; d < VE; ++d) o[d] = 0.f;
  for (int c0 = 0; c0 < w.chunks; c0 += 64) {
    const bool on = c0 + lane < w.chunks;
    const float2 x = ml[min(c0 + lane, w.chunks - 1) * next];
    float wt = 0.f;
    for (int j0 = 0; j0 < min(64, w.chunks - c0); j0 += 4 * AHEAD) {
      f32x4_v y[AHEAD][VE / 4];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
#pragma unroll
        for (int d = 0; d < VE / 4; ++d) y[i][d] = *(const f32x4_v *)(part + min(c0 + j0 + 4 * i + quarter, w.chunks - 1) * next * HD + 4 * d);
      if (j0 == 0) {  // (behind the first loads)
        const float mn = fmaxf(m, wave_max(on ? x.x : -INFINITY)), was = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.sl2);
        wt = !on || x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x.x - mn) * a.sl2);
        m = mn;
        l = l * was + wave_sum(on ? x.y * wt : 0.f);
#pragma unroll
        for (int d = 0; d < VE; ++d) o[d] *= was;
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int j = j0 + 4 * i + quarter;
        const float wj = __shfl(wt, j, 64);
#pragma unroll
        for (int d = 0; d < VE; ++d) o[d] += c0 + j < w.chunks ? y[i][d / 4][d % 4] * wj : 0.f;
      }
    }
  }
#pragma unroll
  for (int other = 16; other <= 32; other <<= 1) {
#pragma unroll
    for (int d = 0; d < VE; ++d) o[d] += __shfl_xor(o[d], other, 64);
  }
  if (quarter) return;
  const bool none = nothing_seen(m, l);
  const float inv = 1.f / l;
  const int i = f / a.G;
  T *dst = (T *)a.out + (s.row0 + i) * a.out_stride + (hk * a.G + f - i * a.G) * HD + d0;
#pragma unroll
  for (int d = 0; d < VE; ++d) Conv<T>::st(dst, d, none ? 0.f : o[d] * inv);
}

// ------------------------------------------------------------------ launch
struct Shape {
  int qt, R, align, slots;             // slots: workgroups per key head that fill the chip
  int64_t tiles, units, cut, parts;    // per key head, at most: tiles, chunks, tiles that are cut, their chunks
  bool whole;                          // no tile is cut
};

// Query rows of a tile: as few as hold a sequence's, since a tile reads the cache once for all of its rows.  Beyond 64 rows 128, or 256
// where these make two rounds of workgroups and more.  us with 128 and with 256, bf16, 32 heads over 8: six sequences of 1000 rows (768 tiles of 256)
// over up to 8192 positions 702 and 652 with heads of 128, 409 and 409 with heads of 64; one of 1500 (192 tiles) over 2048 positions
// 68 and 66, 40 and 47; over 8192 253 and 219, 148 and 153.  So with few tiles heads of 64 gain from 128, heads of 128 would not need them.
// (All figures here are of caches of 16 bits.  One of 8 goes by the same rules; its own sides were not measured.)
static Shape attend_shape(const spec_paged_cache *c, const spec_paged_batch *b, int n_q, int window) {
  Shape s{};
  const int64_t Hk = c->n_kv_heads, G = n_q / Hk, per = (int64_t)b->max_rows * G;
  auto tiles = [&](int R) { return std::min((int64_t)b->B * ((per + R - 1) / R), (int64_t)b->rows * G / R + b->B); };
  const bool f32 = c->dtype == SPEC_DTYPE_F32;
  s.qt = per <= 16 && !(f32 && c->head_dim == 128) ? 1 : per <= 32 || f32 ? 2 : per <= 64 ? 4 : tiles(256) * Hk < 512 ? 8 : 16;
  s.R = 16 * s.qt;
  s.align = s.qt < 8 ? 128 : s.R * 64 / c->head_dim;
  s.tiles = tiles(s.R);
  s.slots = std::max(1, 256 * attend_resident((int)dtype_bytes(c->dtype), c->head_dim, s.qt) / (int)Hk);
  // What a tile can need at most decides whether any is cut, and so whether there is a second kernel, which costs a launch and the search for its work
  // even where it finds nothing to join.  us without cutting and with it, bf16, heads of 128.  One row of 64 sequences, 32 heads over 8: up to 1536 positions
  // 67 and 77, up to 4096 164 and 174; of one sequence: 768 positions 11 and 11, 1536 18 and 12, 4096 43 and 16.  So many sequences pay 5 to 20 %
  // for the second kernel, and few gain from it below the limit already.  Chunks of rows: 100 of one sequence over 448 positions 20 and 22, over
  // 1024 35 and 27; 400 of eight sequences (832 tiles) over up to 2048 113 and 116; 300 of four (320 tiles) over up to 2048 71 and 104,
  // over up to 3000 95 and 75.
  const int64_t span = window ? std::min<int64_t>(b->max_len, (int64_t)window + (s.R - 1) / G + 32) : b->max_len;
  s.whole = span <= (s.qt < 8 ? 1536 : s.tiles * Hk >= 256 ? 2048 : 512);
  s.units = s.tiles + (s.whole ? 0 : s.slots);
  s.cut = s.whole ? 0 : std::min<int64_t>(s.tiles, s.slots * 2 / 3 + 1);
  s.parts = s.whole ? 0 : s.slots * 4 / 3 + 2;
  return s;
}
static size_t attend_bytes(const spec_paged_cache *c, const Shape &s) {
  return (size_t)s.parts * c->n_kv_heads * s.R * (c->head_dim + 2) * sizeof(float);
}
// (behind paged_args)
static int attend_check(const char *who, const spec_paged_cache *c, const spec_paged_batch *b, int n_q, int window, AttendArgs &a, Shape &s) {
  if (n_q < 1 || n_q % c->n_kv_heads)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: n_q_heads=%d is not a multiple of n_kv_heads=%d", who, n_q, c->n_kv_heads);
  a.G = n_q / c->n_kv_heads;
  if ((int64_t)b->rows * a.G >= 1 << 30) return fail_noctx(SPEC_ERR_CAPACITY, "%s: more than 2^30 query rows of a key head", who);
  if (b->B == 0 || b->rows == 0) { s = Shape{};  return SPEC_OK; }
  s = attend_shape(c, b, n_q, window);
  if (s.units * c->n_kv_heads * 512 >= (int64_t)1 << 32)
    return fail_noctx(SPEC_ERR_CAPACITY, "%s: %lld tiles of %d key heads are beyond one launch", who, (long long)s.units, c->n_kv_heads);
  return SPEC_OK;
}

// More LDS than 64 KB has to be asked for, once on every device.
template <class Sb, class Sh> static hipError_t allow_chunk_lds() {
  static std::mutex mutex;
  static bool done[64];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  std::lock_guard<std::mutex> lock(mutex);
  if (dev >= 0 && dev < 64 && done[dev]) return hipSuccess;
  const void *kernels[4] = {(const void *)k_paged_chunk<bf16_t, Sb, 64, 8>, (const void *)k_paged_chunk<bf16_t, Sb, 128, 8>,
                            (const void *)k_paged_chunk<f16_t, Sh, 64, 8>, (const void *)k_paged_chunk<f16_t, Sh, 128, 8>};
  for (const void *k : kernels) {
    e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, pc_lds(8));
    if (e != hipSuccess) return e;
  }
  if (dev >= 0 && dev < 64) done[dev] = true;
  return hipSuccess;
}

template <class T, class S, int HD, int QT>
static void attend_launch(const AttendArgs &a, const Shape &s, hipStream_t st) {
  const int64_t groups = s.units * a.p.n_kv_heads;
  const dim3 grid((unsigned)(sizeof(S) == 1 && QT < 8 ? (groups + 63) / 64 * 64 : groups));
  if constexpr (QT >= 8) hipLaunchKernelGGL((k_paged_chunk<T, S, HD, QT / 2>), grid, dim3(32 * QT), pc_lds(QT / 2), st, a);
  else hipLaunchKernelGGL((k_paged_attend<T, S, HD, QT>), grid, dim3(256), 0, st, a);
  if (!s.cut) return;
  if constexpr (sizeof(S) == 1 && QT < 8)
    hipLaunchKernelGGL((k_paged_join_rows<T, HD, QT>), dim3((unsigned)(s.cut * a.p.n_kv_heads * 4 * QT)), dim3(256), 0, st, a, s.align);
  else hipLaunchKernelGGL((k_paged_join<T, HD, QT>), dim3((unsigned)(s.cut * a.p.n_kv_heads * QT)), dim3(256), 0, st, a, s.align);
}

// A call: checked, with its arguments in `a` and its shape in `s`, behind paged_args.  nothing: there is no work.
static int attend_prepare(const char *who, const spec_paged_cache *cache, const spec_paged_batch *batch, int n_q_heads, const void *d_q,
                          int64_t q_stride, float scale, int window, void *d_workspace, size_t workspace_bytes, void *d_out, int64_t out_stride,
                          AttendArgs &a, Shape &s, bool &nothing) {
  // A window that reaches over all positions is none.  (So a window is at most 2^30, and its differences with positions stay inside 32 bits, those
  // of dead rows as well.)
  const bool endless = window >= batch->max_len;
  int rc = attend_check(who, cache, batch, n_q_heads, endless ? 0 : std::max(window, 0), a, s);
  if (rc) return rc;
  a.sl2 = scale * 1.4426950408889634f;
  if (!(scale > 0.f) || std::isinf(a.sl2)) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: scale must be positive and below 2.3e38", who);
  if (window < 0) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: window=%d", who, window);
  nothing = batch->B == 0 || batch->rows == 0;
  if (nothing) return SPEC_OK;
  if ((rc = paged_rows_check(who, "d_q", cache, n_q_heads, d_q, q_stride))) return rc;
  if ((rc = paged_rows_check(who, "d_out", cache, n_q_heads, d_out, out_stride))) return rc;
  const size_t need = attend_bytes(cache, s);
  if (need && (!d_workspace || ((uintptr_t)d_workspace & 255) || workspace_bytes < need))
    return fail_noctx(SPEC_ERR_WORKSPACE, "%s: workspace null, not 256-byte aligned, or smaller than %zu bytes", who, need);
  a.q = (const unsigned char *)d_q;
  a.out = (unsigned char *)d_out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.window = endless ? 0 : window;
  a.part = (float *)d_workspace;
  a.ml = need ? a.part + (size_t)s.parts * cache->n_kv_heads * s.R * cache->head_dim : nullptr;
  a.chunk_min = s.whole ? 1 << 30 : PA_CHUNK_MIN;
  a.one_slot = 1.f / s.slots;
  return SPEC_OK;
}
template <class T, class S>
static void attend_dispatch(int head_dim, const AttendArgs &a, const Shape &s, hipStream_t st) {
  auto of = [&](auto HD_) {
    constexpr int HD = decltype(HD_)::value;
    if (s.qt == 1) {
      if constexpr (sizeof(T) == 2 || HD == 64) attend_launch<T, S, HD, 1>(a, s, st);
    } else if (s.qt == 2) attend_launch<T, S, HD, 2>(a, s, st);
    else if constexpr (sizeof(T) == 2) {
      if (s.qt == 4) attend_launch<T, S, HD, 4>(a, s, st);
      else if (s.qt == 8) attend_launch<T, S, HD, 8>(a, s, st);
      else attend_launch<T, S, HD, 16>(a, s, st);
    }
  };
  if (head_dim == 64) of(std::integral_constant<int, 64>{});
  else of(std::integral_constant<int, 128>{});
}

}  // namespace spec
