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
//
// Chunks: a sequence with more rows or positions has more work, and the host does not know the lengths.  Every wave adds the
// batch's work up (a load and a few shuffles) and derives from it how long a chunk is: as many chunks as fill the chip's slots
// evenly, whatever the lengths are.
#include "paged.h"
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
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_v;

constexpr int PA_SLOTS = 1024;    // workgroups that a pass is cut into where it is long enough
constexpr int PC_SLOTS = 2048;    // the same for tiles of many rows
constexpr int PA_CHUNK_MIN = 512; // positions of the shortest chunk: a shorter context is not worth a second kernel
constexpr int PA_WAVES = 4;

struct AttendArgs {
  PagedArgs p;
  const unsigned char *q;
  unsigned char *out;
  int64_t q_stride, out_stride;  // elements
  int G, window;
  float sl2;                     // scale * log2(e)
  float *part, *ml;              // [unit * heads][R][HD], [unit * heads][R][2]
  int slots;                     // workgroups per key head that the work is cut into
};

// ------------------------------------------------------------------ work
struct Work { int b, tile, chunk, chunks, base, chunk_len; PagedSeq s; };
__device__ __forceinline__ Work in_scalars(const Work &w) {
  auto f = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  return Work{f(w.b), f(w.tile), f(w.chunk), f(w.chunks), f(w.base), f(w.chunk_len), PagedSeq{f(w.s.row0), f(w.s.n), f(w.s.kv)}};
}

__device__ __forceinline__ int seq_tiles(const AttendArgs &a, const PagedSeq &s, int R) { return (s.n * a.G + R - 1) / R; }
// positions that a tile of the sequence can need, at most
__device__ __forceinline__ int seq_span(const AttendArgs &a, const PagedSeq &s, int R) {
  if (!a.window) return s.kv;
  return (int)min((int64_t)s.kv, (int64_t)a.window + (R - 1) / a.G + 32);
}
template <class V>
__device__ __forceinline__ V wave_scan(V v) {  // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const V t = __shfl_up(v, o, 64);
    if ((int)(threadIdx.x & 63) >= o) v += t;
  }
  return v;
}

// Unit `unit` of the pass's work: a chunk of a tile (TILES false), or a tile (TILES true; base is then its first chunk's unit).  The
// same for the whole wave; false: there is none.
template <bool TILES>
__device__ __forceinline__ bool find_work(const AttendArgs &a, int R, int unit, Work &w) {
  const int lane = threadIdx.x & 63, per = (a.p.B + 63) / 64, first = lane * per, last = min(a.p.B, first + per);
  PagedSeq s{};
  long long sum = 0;
  for (int b = first; b < last; ++b) {
    s = paged_seq(a.p, b);
    sum += (long long)seq_tiles(a, s, R) * seq_span(a, s, R);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  const long long even = (sum + a.slots - 1) / a.slots;
  const int len = max(PA_CHUNK_MIN, (int)min((even + 127) / 128 * 128, (long long)1 << 30));
  int units = 0, tiles = 0;
  for (int b = first; b < last; ++b) {
    if (per > 1) s = paged_seq(a.p, b);
    const int t = seq_tiles(a, s, R);
    tiles += t;
    units += t * max(1, (seq_span(a, s, R) + len - 1) / len);
  }
  const int units_to = wave_scan(units), tiles_to = TILES ? wave_scan(tiles) : 0;
  const int to = TILES ? tiles_to : units_to, mine = TILES ? tiles : units;
  const unsigned long long here = __ballot(unit >= to - mine && unit < to);
  if (!here) return false;
  const int src = __builtin_ctzll(here);
  int at = __shfl(to - mine, src, 64), base = __shfl(units_to - units, src, 64);
  for (int b = src * per; b < min(a.p.B, src * per + per); ++b) {
    if (per > 1) {
      s = paged_seq(a.p, b);
    } else {
      s.row0 = __shfl(s.row0, src, 64); s.n = __shfl(s.n, src, 64); s.kv = __shfl(s.kv, src, 64);
    }
    const int t = seq_tiles(a, s, R), c = max(1, (seq_span(a, s, R) + len - 1) / len), n = TILES ? t : t * c;
    if (unit < at + n) {
      const int u = unit - at;
      w.b = b;
      w.chunks = c;
      // the last rows of a sequence see the most: their tiles start first
      w.tile = TILES ? t - 1 - u : t - 1 - u % t;
      w.chunk = TILES ? 0 : u / t;
      w.base = TILES ? base + u : 0;  // the tile's chunk j is unit base + j * tiles
      w.chunk_len = len;
      w.s = s;
      return true;
    }
    at += n;
    base += t * c;
  }
  return false;
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

// A lane's part of a step: its key rows of the two key tiles (KU units of 16 bytes each, units 4 kk + g), and 8 positions of
// VE = HD / 16 values, as loaded.
template <class T, int HD> struct Step {
  static constexpr int E = 16 / sizeof(T), KU = HD / (4 * E), VE = HD / 16, VW = VE * sizeof(T) / 4;  // VW: words of a position's values
  u32x4_v k0[KU], k1[KU];
  uint32_t v[8][VW];
};

template <class T, int HD>
__device__ __forceinline__ void load_step(Step<T, HD> &f, const PagedArgs &p, size_t head_at, int page_k, int page_v, int ks, int r, int g) {
  constexpr int VW = Step<T, HD>::VW;
  const size_t pos_bytes = (size_t)p.pos_units << 4;
  // an absent page's loads go to page 0, which exists; what they bring is not used
  const unsigned char *kr = p.k + head_at + 16 * g + paged_row(p, max(page_k, 0), ks + 8 * (r >> 2) + (r & 3));
#pragma unroll
  for (int kk = 0; kk < Step<T, HD>::KU; ++kk) {
    f.k0[kk] = *(const u32x4_v *)(kr + 64 * kk);
    f.k1[kk] = *(const u32x4_v *)(kr + 4 * pos_bytes + 64 * kk);
  }
  const unsigned char *vr = p.v + head_at + 4 * VW * r + paged_row(p, max(page_v, 0), ks + 8 * g);
#pragma unroll
  for (int i = 0; i < 8; ++i) __builtin_memcpy(f.v[i], __builtin_assume_aligned(vr + i * pos_bytes, VW * 4 < 16 ? VW * 4 : 16), VW * 4);
}

// S^T of a step: s0[i] <-> key 8g + i, s1[i] <-> key 8g + 4 + i of lane (query r, g)
template <class T, int HD>
__device__ __forceinline__ void scores(const Step<T, HD> &f, const u32x4_v (&q)[Step<T, HD>::KU], float (&sv)[8]) {
  f32x4_v s0 = (f32x4_v){0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
  for (int kk = 0; kk < Step<T, HD>::KU; ++kk) {
    if constexpr (sizeof(T) == 2) {
      s0 = Mat<T>::run(f.k0[kk], q[kk], s0);
      s1 = Mat<T>::run(f.k1[kk], q[kk], s1);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f.k0[kk][i]), __uint_as_float(q[kk][i]), s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f.k1[kk][i]), __uint_as_float(q[kk][i]), s1, 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { sv[i] = s0[i]; sv[4 + i] = s1[i]; }
}

// the 8 positions of element ht of a lane's values, as an operand
template <class T, int HD>
__device__ __forceinline__ u32x4_v value_operand(const Step<T, HD> &f, int ht) {
  u32x4_v x;
#pragma unroll
  for (int d = 0; d < 4; ++d)
    x[d] = __builtin_amdgcn_perm(f.v[2 * d + 1][ht / 2], f.v[2 * d][ht / 2], (ht & 1) ? 0x07060302u : 0x05040100u);
  return x;
}

// Takes infinities and NaN out of a word of cached values; whether there were any.
template <class T> __device__ __forceinline__ bool drop_odd(uint32_t &w) {
  constexpr uint32_t e = sizeof(T) == 4 ? 0x7f800000u : std::is_same<T, bf16_t>::value ? 0x7f80u : 0x7c00u;
  const bool lo = (w & e) == e, hi = sizeof(T) == 2 && (w >> 16 & e) == e;
  if (sizeof(T) == 4) w = lo ? 0u : w;
  else w &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  return lo || hi;
}
// The value if it is infinite or NaN, else zero.
template <class T> __device__ __forceinline__ float only_odd(T t) {
  const float v = Conv<T>::ld(&t, 0);
  return fabsf(v) < INFINITY ? 0.f : v;
}

// ------------------------------------------------------------------ few query rows a tile: the waves share the positions
template <class T, int HD, int QT>
__global__ __launch_bounds__(256) void k_paged_attend(AttendArgs a) {
  typedef Step<T, HD> St;
  constexpr int R = 16 * QT, HT = HD / 16, KU = St::KU, VE = St::VE, LD = HD + 4;
  constexpr bool AHEAD = QT * HD * (int)sizeof(T) < 1024;  // registers for the next step's loads beside this step's
  __shared__ float sh_o[PA_WAVES][16][LD];
  __shared__ float sh_m[PA_WAVES][R], sh_l[PA_WAVES][R];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int Hk = a.p.n_kv_heads, unit = blockIdx.x / Hk, hk = blockIdx.x % Hk;
  Work w;
  if (!find_work<false>(a, R, unit, w)) return;
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
    const T *src = (const T *)a.q + (on ? (s.row0 + i) * a.q_stride + (hk * a.G + f - i * a.G) * HD : 0) + g * St::E;
#pragma unroll
    for (int kk = 0; kk < KU; ++kk) q[t][kk] = on ? *(const u32x4_v *)(src + kk * 4 * St::E) : (u32x4_v){0, 0, 0, 0};
  }
  // every row of the tile sees all positions [see_lo, see_hi)
  const int i0 = w.tile * R / a.G, i1 = min(s.n - 1, (w.tile * R + R - 1) / a.G);
  const int see_hi = s.kv - s.n + i0 + 1, see_lo = a.window ? s.kv - s.n + i1 - a.window + 1 : 0;

  float m[QT], l[QT];
  f32x4_v acc[QT][HT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) acc[t][ht] = (f32x4_v){0.f, 0.f, 0.f, 0.f};
  }

  const size_t head_at = (size_t)hk * a.p.head_units << 4;  // bytes
  // Pages of 16 of the wave's steps at a time: lane 4j + i holds that of the i-th eight positions of step j.
  const int ks0 = k_begin + 32 * wv;
  auto pages_at = [&](int ks) {
    const int pos = ks + 128 * (lane >> 2) + 8 * (lane & 3);
    return pos < k_end ? paged_page(a.p, w.b, pos) : -1;
  };
  int pages = -1, pages_next = -1;
  St cur, nxt;
  int pk = -1, pv = -1, pk_n = -1, pv_n = -1;
  if (ks0 < k_end) {
    pages = pages_at(ks0);
    pages_next = pages_at(ks0 + 16 * 128);
    pk = __shfl(pages, r >> 2, 64);
    pv = __shfl(pages, g, 64);
    load_step<T, HD>(cur, a.p, head_at, pk, pv, ks0, r, g);
  }
  int j = 0;
  bool odd = false;
  for (int ks = ks0; ks < k_end; ks += 128) {
    if (ks + 128 < k_end) {
      if (++j == 16) {
        j = 0;
        pages = pages_next;
        pages_next = pages_at(ks + 128 + 16 * 128);
      }
      pk_n = __shfl(pages, 4 * j + (r >> 2), 64);
      pv_n = __shfl(pages, 4 * j + g, 64);
      if (AHEAD) load_step<T, HD>(nxt, a.p, head_at, pk_n, pv_n, ks + 128, r, g);
    }
    // keys of this lane's scores: ks + 8g + i, in page pv
    const bool whole = ks >= see_lo && ks + 32 <= min(see_hi, k_end) && __all(pv >= 0);
    if (!whole) {  // positions that no row of the tile sees: their values, whatever they are, become zeros
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool live = pv >= 0 && ks + 8 * g + i < k_end && ks + 8 * g + i >= 0;
#pragma unroll
        for (int x = 0; x < St::VW; ++x) cur.v[i][x] = live ? cur.v[i][x] : 0u;
      }
    }
    // Positions that some of the tile's rows see and others do not: a weight of zero does not keep an infinity or a NaN out of a
    // product, so such values leave here and are added at the end for the rows that see them.
    if (!whole && i0 != i1) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int x = 0; x < St::VW; ++x) odd |= drop_odd<T>(cur.v[i][x]);
    }
    float p[QT][8];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float sv[8];
      scores<T, HD>(cur, q[t], sv);
      if (!whole) {
        const int from = a.window ? pos[t] - a.window + 1 : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = ks + 8 * g + i;
          sv[i] = pv >= 0 && key <= pos[t] && key >= from && key < k_end ? sv[i] : -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (__any(top > m[t])) {
        const float mn = fmaxf(m[t], top);
        const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[t] - mn) * a.sl2);
        m[t] = mn;
        l[t] *= corr;
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) { acc[t][ht][0] *= corr; acc[t][ht][1] *= corr; acc[t][ht][2] *= corr; acc[t][ht][3] *= corr; }
      }
      const float off = m[t] == -INFINITY ? 0.f : m[t] * a.sl2;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[t][i] = __builtin_amdgcn_exp2f(fmaf(sv[i], a.sl2, -off));
        l[t] += p[t][i];
      }
    }
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) {
      if constexpr (sizeof(T) == 2) {
        const u32x4_v x = value_operand<T, HD>(cur, ht);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          u32x4_v y;
#pragma unroll
          for (int d = 0; d < 4; ++d) y[d] = Mat<T>::pack2(p[t][2 * d], p[t][2 * d + 1]);
          acc[t][ht] = Mat<T>::run(x, y, acc[t][ht]);
        }
      } else {
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            acc[t][ht] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(cur.v[i][ht]), p[t][i], acc[t][ht], 0, 0, 0);
      }
    }
    if (AHEAD) cur = nxt;
    else if (ks + 128 < k_end) load_step<T, HD>(cur, a.p, head_at, pk_n, pv_n, ks + 128, r, g);
    pv = pv_n;
  }

  if (__any(odd)) {  // this wave's steps of the positions outside [see_lo, see_hi) again
    for (int ks = ks0; ks < k_end; ks += 128) {
      if (ks >= see_lo && ks + 32 <= min(see_hi, k_end)) continue;
      for (int key = ks; key < min(ks + 32, k_end); ++key) {
        const int page = paged_page(a.p, w.b, key);
        if (page < 0) continue;
        const T *src = (const T *)(a.p.v + head_at + paged_row(a.p, page, key)) + 4 * VE * g;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          if (key > pos[t] || (a.window && key <= pos[t] - a.window)) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) acc[t][ht][e] += only_odd<T>(src[VE * e + ht]);
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
  const int64_t slot = (int64_t)blockIdx.x * R;
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
        const float inv = lr == 0.f ? 0.f : 1.f / lr;
        const int i = f / a.G;
        T *dst = (T *)a.out + (s.row0 + i) * a.out_stride + (hk * a.G + f - i * a.G) * HD + d0;
#pragma unroll
        for (int d = 0; d < VE; ++d) Conv<T>::st(dst, d, lr == 0.f ? 0.f : o[d] * inv);
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
// The largest of 16.  Written as fmaxf, every score is first brought to canonical form by an instruction of its own.
__device__ __forceinline__ float max16(const f32x16_v &x) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3\n\tv_max3_f32 %0, %0, %4, %5\n\tv_max3_f32 %0, %0, %6, %7\n\tv_max3_f32 %0, %0, %8, %9\n\t"
      "v_max3_f32 %0, %0, %10, %11\n\tv_max3_f32 %0, %0, %12, %13\n\tv_max3_f32 %0, %0, %14, %15\n\tv_max_f32 %0, %0, %16"
      : "=&v"(r)
      : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]), "v"(x[8]), "v"(x[9]), "v"(x[10]), "v"(x[11]),
        "v"(x[12]), "v"(x[13]), "v"(x[14]), "v"(x[15]));
  return r;
}
__device__ __forceinline__ float max_of_halves(float v) { return fmaxf(v, __shfl_xor(v, 32, 64)); }

// A workgroup of NW waves takes 32 NW query rows, 32 a wave, and walks the positions in tiles of KT = 16 NW (heads of 128) or 32 NW (of 64):
// 4 NW KB of keys and as much of values, in LDS in operand order, twice.  32x32x16 products: a lane owns one query (lane % 32) and half of
// every 16 keys, so a row's maximum takes one exchange.  Keys go straight to LDS, [key][unit of 16 bytes], a row's units exchanged by its number so
// that reading one unit of 32 rows meets every bank; of values a thread loads 8 positions of 4 elements and turns them round on
// the way to LDS.  The maximum follows the scores only when they have grown
// by 2^8: weights up to 2^8 are as exact in 16 bits as weights up to 1, the sums are fp32, and most tiles then rescale nothing.
constexpr int pc_lds(int NW) { return 4 * NW * 256 * 16; }

template <class T, int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_paged_chunk(AttendArgs a) {
  constexpr int R = 32 * NW, NC = HD / 8, KK = HD / 16, DT = HD / 32, KT = 256 * NW / NC, VC = HD / 4, IPT = 32 / VC, UNITS = KT * NC;
  extern __shared__ __attribute__((aligned(16))) u32x4_v pc_smem[];  // [2] keys [KT][NC], [2] values [KT / 16][DT][2][32]
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const int Hk = a.p.n_kv_heads, unit = blockIdx.x / Hk, hk = blockIdx.x % Hk;
  Work w;
  if (!find_work<false>(a, R, unit, w)) return;
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
  const unsigned char *k_base = a.p.k + head_at, *v_base = a.p.v + head_at + 8 * vc;
  const int32_t *table = a.p.pages + w.b * a.p.pages_stride;
  const size_t pos_bytes = (size_t)a.p.pos_units << 4;
  auto page_at = [&](int pos) {  // of a position before k_end; behind it, the last one's
    const int page = table[(unsigned)min(pos, k_end - 1) >> a.p.page_shift];
    return (unsigned)page < (unsigned)a.p.n_pages ? page : -1;
  };
  // Row 32 u + 16 x + 8 y + 4 z + e of a key tile holds key 32 u + 16 x + 8 z + 4 y + e.  Wave instruction `it` fills 64 / NC rows; its
  // lanes' keys lie in one of two groups of eight positions, kgrp[it's].
  const int kgrp0 = NC == 16 ? 2 * wv : 4 * wv + (lane >> 5), kgrp1 = kgrp0 + (NC == 16 ? 1 : 2);
  const int krow = NC == 16 ? 16 * wv + (lane >> 4) : 32 * wv + 8 * (lane >> 5) + (lane >> 3 & 3);  // key of it = 0
  uint32_t x[8][2];
  int x_page;
  struct Pages { int k[2], v; };
  auto pages_of = [&](int ks) { return Pages{{page_at(ks + 8 * kgrp0), page_at(ks + 8 * kgrp1)}, page_at(ks + 8 * kg)}; };
  auto fetch = [&](int ks, const Pages &pg, int kbuf) {
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int key = krow + (NC == 16 ? 8 * (it & 1) + 4 * (it >> 1) : 16 * (it >> 1) + 4 * (it & 1));
      const int unit = NC == 16 ? (lane ^ (lane >> 4)) % 16 ^ 4 * it : (lane ^ (lane >> 3)) % 8;  // by the row's number
      const unsigned char *src = k_base + paged_row(a.p, max(pg.k[NC == 16 ? it & 1 : it >> 1], 0), ks + key) + 16 * unit;
      lanes_to_lds(src, (unsigned)((kbuf * UNITS + (wv * 4 + it) * 64) * 16));
    }
    const unsigned char *src = v_base + paged_row(a.p, max(pg.v, 0), ks + 8 * kg);
    x_page = pg.v;
#pragma unroll
    for (int i = 0; i < 8; ++i) __builtin_memcpy(x[i], __builtin_assume_aligned(src + i * pos_bytes, 8), 8);
  };
  // Positions that some of the tile's rows see and others do not (those outside [all_lo, all_hi)): a weight of zero does not keep an infinity
  // or a NaN out of a product, so such values leave here and are added at the end for the rows that see them.
  const int all_hi = p0 + w.tile * R / a.G + 1, all_lo = a.window ? p0 + min(w.tile * R + R - 1, rows - 1) / a.G - a.window + 1 : 0;
  bool odd = false;
  auto store = [&](int ks, int vbuf) {
    const int live = x_page < 0 ? 0 : k_end - (ks + 8 * kg);  // positions behind the end hold anything
    if (live < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i][0] = i < live ? x[i][0] : 0u; x[i][1] = i < live ? x[i][1] : 0u; }
    }
    if (ks + KT > all_hi || ks < all_lo) {
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
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  float m = -INFINITY, l = 0.f;
  const float grow = 8.f / a.sl2;
  f32x16_v acc[DT];
#pragma unroll
  for (int j = 0; j < DT; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;

  // score e of sc[u]: key ks + 32 u + 16 (e / 8) + 8 h + e % 8
  f32x16_v sc[2];
  auto key_products = [&](const u32x4_v *kb) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) sc[u] = mat32<T>(kb[(32 * u + col) * NC + ((2 * kk + h) ^ (col & (NC - 1)))], q[kk], sc[u]);
    }
  };
  // the maximum follows where it has to; -> what is taken off the scaled scores
  auto follow = [&]() {
    const float top = max_of_halves(fmaxf(max16(sc[0]), max16(sc[1])));
    if (__any(top > m + grow)) {
      const float mn = fmaxf(m, top), corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.sl2);
      m = mn;
      l *= corr;
#pragma unroll
      for (int j = 0; j < DT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][e] *= corr;
    }
    return m == -INFINITY ? 0.f : m * a.sl2;
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
  auto there_at = [&](int ks) { return lane < KT / 8 ? page_at(ks + 8 * lane) : -1; };
  unsigned present = 0;
  Pages pages{{-1, -1}, -1};
  if (k_begin < k_end) {
    const int there = there_at(k_begin);
    fetch(k_begin, pages_of(k_begin), 0);
    pages = pages_of(k_begin + KT);
    store(k_begin, 0);
    present = (unsigned)__ballot(there >= 0);
  }
  meet();
  int buf = 0;
  for (int ks0 = k_begin; ks0 < k_end; ks0 += KT, buf ^= 1) {
    // The next tile's loads land while this one is worked on.  Behind the last tile they bring page 0's rows, which nothing reads: no branch
    // keeps the address arithmetic from the products' shadow.
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
      const float off = follow();
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const u32x4_v p = weights(y, off);
#pragma unroll
        for (int j = 0; j < DT; ++j) acc[j] = mat32<T>(vs[(y * DT + j) * 64], p, acc[j]);
      }
    }
    store(ks0 + KT, buf ^ 1);
    present = (unsigned)__ballot(there >= 0);
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
      if (key >= all_lo && key < all_hi) { key = all_hi - 1; continue; }
      const int page = page_at(key);
      if (page < 0 || key > pos || key < from) continue;
      const T *src = (const T *)(a.p.v + head_at + paged_row(a.p, page, key));
#pragma unroll
      for (int j = 0; j < DT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int row = 8 * (e >> 2) + 4 * h + (e & 3);
          acc[j][e] += only_odd<T>(src[4 * (row % VC) + j * IPT + row / VC]);
        }
    }
  }
  if (!on) return;
  // element 4 c + i of the query lies in tile i / IPT, row c + VC (i % IPT); a lane holds the rows 8 (e / 4) + 4 h + e % 4
  const bool several = w.chunks > 1;
  const int64_t at = (int64_t)blockIdx.x * R + 32 * wv + col;
  const float inv = l == 0.f ? 0.f : 1.f / l;
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
        for (int i = 0; i < 4; ++i) v[i] = Mat<T>::pack2(l == 0.f ? 0.f : o[8 * y + 2 * i] * inv, l == 0.f ? 0.f : o[8 * y + 2 * i + 1] * inv);
        *(u32x4_v *)(dst + d + 8 * y) = v;
      }
    }
  }
}

// Joins the chunks of a tile: a workgroup takes 16 query rows of a tile, a thread VE elements of one.
template <class T, int HD, int QT>
__global__ __launch_bounds__(256) void k_paged_join(AttendArgs a) {
  constexpr int R = 16 * QT, VE = HD / 16;
  const int Hk = a.p.n_kv_heads, id = blockIdx.x / QT, t = blockIdx.x % QT, unit = id / Hk, hk = id % Hk;
  Work w;
  if (!find_work<true>(a, R, unit, w) || w.chunks < 2) return;
  const PagedSeq s = w.s;
  const int row = threadIdx.x >> 4, d0 = VE * (threadIdx.x & 15), f = w.tile * R + 16 * t + row;
  if (f >= s.n * a.G) return;
  const int tiles = seq_tiles(a, s, R);
  float m = -INFINITY, l = 0.f, o[VE];
#pragma unroll
  for (int d = 0; d < VE; ++d) o[d] = 0.f;
  for (int c = 0; c < w.chunks; ++c) {
    const int64_t at = ((int64_t)(w.base + c * tiles) * Hk + hk) * R + 16 * t + row;
    const float mc = a.ml[at * 2], lc = a.ml[at * 2 + 1];
    const float mn = fmaxf(m, mc);
    const float wa = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.sl2);
    const float wb = mc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mc - mn) * a.sl2);
    l = l * wa + lc * wb;
#pragma unroll
    for (int d = 0; d < VE; ++d) o[d] = o[d] * wa + a.part[at * HD + d0 + d] * wb;
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int i = f / a.G;
  T *dst = (T *)a.out + (s.row0 + i) * a.out_stride + (hk * a.G + f - i * a.G) * HD + d0;
#pragma unroll
  for (int d = 0; d < VE; ++d) Conv<T>::st(dst, d, l == 0.f ? 0.f : o[d] * inv);
}

// ------------------------------------------------------------------ launch
struct Shape { int qt, R, slots; int64_t tiles, units; bool join; };

// Query rows of a tile: as few as hold a sequence's, since a tile reads the cache once for all of its rows.
static Shape attend_shape(const spec_paged_cache *c, const spec_paged_batch *b, int n_q) {
  Shape s;
  const int64_t G = n_q / c->n_kv_heads, per = (int64_t)b->max_rows * G;
  s.qt = per <= 16 ? 1 : per <= 32 || c->dtype == SPEC_DTYPE_F32 ? 2 : per <= 64 ? 4 : per <= 128 ? 8 : 16;
  s.R = 16 * s.qt;
  s.tiles = std::min((int64_t)b->B * ((per + s.R - 1) / s.R), (int64_t)b->rows * G / s.R + b->B);
  s.join = b->max_len > PA_CHUNK_MIN;
  s.slots = std::max(1, (s.qt >= 8 ? PC_SLOTS * 8 / s.qt : PA_SLOTS) / c->n_kv_heads);
  s.units = s.tiles + (s.join ? s.slots : 0);
  return s;
}
static size_t attend_bytes(const spec_paged_cache *c, const Shape &s) {
  return s.join ? (size_t)s.units * c->n_kv_heads * s.R * (c->head_dim + 2) * sizeof(float) : 0;
}
static int attend_check(const char *who, const spec_paged_cache *c, const spec_paged_batch *b, int n_q, AttendArgs &a, Shape &s) {
  int rc = paged_args(who, c, b, &a.p);
  if (rc) return rc;
  if (n_q < 1 || n_q % c->n_kv_heads)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: n_q_heads=%d is not a multiple of n_kv_heads=%d", who, n_q, c->n_kv_heads);
  a.G = n_q / c->n_kv_heads;
  if ((int64_t)b->rows * a.G >= 1 << 30) return fail_noctx(SPEC_ERR_CAPACITY, "%s: more than 2^30 query rows of a key head", who);
  if (b->B == 0 || b->rows == 0) { s = Shape{1, 16, 1, 0, 0, false}; return SPEC_OK; }
  s = attend_shape(c, b, n_q);
  if (s.units * c->n_kv_heads * 256 >= (int64_t)1 << 32 || s.tiles * c->n_kv_heads * s.qt * 256 >= (int64_t)1 << 32)
    return fail_noctx(SPEC_ERR_CAPACITY, "%s: %lld tiles of %d key heads are beyond one launch", who, (long long)s.units, c->n_kv_heads);
  return SPEC_OK;
}

// More LDS than 64 KB has to be asked for, once on every device.
static hipError_t allow_chunk_lds() {
  static std::mutex mutex;
  static bool done[64];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  std::lock_guard<std::mutex> lock(mutex);
  if (dev >= 0 && dev < 64 && done[dev]) return hipSuccess;
  const void *kernels[4] = {(const void *)k_paged_chunk<bf16_t, 64, 8>, (const void *)k_paged_chunk<bf16_t, 128, 8>,
                            (const void *)k_paged_chunk<f16_t, 64, 8>, (const void *)k_paged_chunk<f16_t, 128, 8>};
  for (const void *k : kernels) {
    e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, pc_lds(8));
    if (e != hipSuccess) return e;
  }
  if (dev >= 0 && dev < 64) done[dev] = true;
  return hipSuccess;
}

template <class T, int HD, int QT>
static void attend_launch(const AttendArgs &a, const Shape &s, hipStream_t st) {
  const dim3 grid((unsigned)(s.units * a.p.n_kv_heads));
  if constexpr (QT >= 8) hipLaunchKernelGGL((k_paged_chunk<T, HD, QT / 2>), grid, dim3(32 * QT), pc_lds(QT / 2), st, a);
  else hipLaunchKernelGGL((k_paged_attend<T, HD, QT>), grid, dim3(256), 0, st, a);
  if (s.join) hipLaunchKernelGGL((k_paged_join<T, HD, QT>), dim3((unsigned)(s.tiles * a.p.n_kv_heads * QT)), dim3(256), 0, st, a);
}

}  // namespace spec

using namespace spec;

extern "C" int spec_paged_attention_workspace_bytes(const spec_paged_cache *cache, const spec_paged_batch *batch, int32_t n_q_heads,
                                                    size_t *bytes) {
  const char *who = "spec_paged_attention_workspace_bytes";
  AttendArgs a{};
  Shape s;
  if (!bytes) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: bytes is null", who);
  const int rc = attend_check(who, cache, batch, n_q_heads, a, s);
  if (rc) return rc;
  *bytes = attend_bytes(cache, s);
  return SPEC_OK;
}

extern "C" int spec_paged_attention(void *hip_stream, const spec_paged_cache *cache, const spec_paged_batch *batch, int32_t n_q_heads,
                                    const void *d_q, int64_t q_stride, float scale, int32_t window, void *d_workspace,
                                    size_t workspace_bytes, void *d_out, int64_t out_stride) {
  const char *who = "spec_paged_attention";
  AttendArgs a{};
  Shape s;
  int rc = attend_check(who, cache, batch, n_q_heads, a, s);
  if (rc) return rc;
  if (!(scale > 0.f) || std::isinf(scale)) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: scale must be positive and finite", who);
  if (window < 0) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: window=%d", who, window);
  if (batch->B == 0 || batch->rows == 0) return SPEC_OK;
  if ((rc = paged_rows_check(who, "d_q", cache, n_q_heads, d_q, q_stride))) return rc;
  if ((rc = paged_rows_check(who, "d_out", cache, n_q_heads, d_out, out_stride))) return rc;
  const size_t need = attend_bytes(cache, s);
  if (need && (!d_workspace || ((uintptr_t)d_workspace & 255) || workspace_bytes < need))
    return fail_noctx(SPEC_ERR_WORKSPACE, "%s: workspace null, not 256-byte aligned, or smaller than %zu bytes", who, need);
  a.q = (const unsigned char *)d_q;
  a.out = (unsigned char *)d_out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.window = window;
  a.sl2 = scale * 1.4426950408889634f;
  a.part = (float *)d_workspace;
  a.ml = need ? a.part + (size_t)s.units * cache->n_kv_heads * s.R * cache->head_dim : nullptr;
  // without a second kernel one chunk holds everything: max_len is at most the shortest chunk
  a.slots = s.slots;
  hipStream_t st = (hipStream_t)hip_stream;
  if (s.qt == 16) {
    const hipError_t e = allow_chunk_lds();
    if (e != hipSuccess) return fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
  }
  SPEC_DISPATCH_DTYPE(cache->dtype, T, {
    if (cache->head_dim == 64) {
      if (s.qt == 1) attend_launch<T, 64, 1>(a, s, st);
      else if (s.qt == 2) attend_launch<T, 64, 2>(a, s, st);
      else if constexpr (sizeof(T) == 2) {
        if (s.qt == 4) attend_launch<T, 64, 4>(a, s, st);
        else if (s.qt == 8) attend_launch<T, 64, 8>(a, s, st);
        else attend_launch<T, 64, 16>(a, s, st);
      }
    } else {
      if (s.qt == 1) attend_launch<T, 128, 1>(a, s, st);
      else if (s.qt == 2) attend_launch<T, 128, 2>(a, s, st);
      else if constexpr (sizeof(T) == 2) {
        if (s.qt == 4) attend_launch<T, 128, 4>(a, s, st);
        else if (s.qt == 8) attend_launch<T, 128, 8>(a, s, st);
        else attend_launch<T, 128, 16>(a, s, st);
      }
    }
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
