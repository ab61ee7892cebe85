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
#include <type_traits>

namespace spec {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_v;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_v;
typedef __attribute__((ext_vector_type(4))) float f32x4_v;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_v;

constexpr int PA_SLOTS = 1024;    // workgroups that a pass is cut into where it is long enough
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
      w.b = __builtin_amdgcn_readfirstlane(b);
      w.chunks = __builtin_amdgcn_readfirstlane(c);
      // the last rows of a sequence see the most: their tiles start first
      w.tile = __builtin_amdgcn_readfirstlane(TILES ? t - 1 - u : t - 1 - u % t);
      w.chunk = __builtin_amdgcn_readfirstlane(TILES ? 0 : u / t);
      w.base = __builtin_amdgcn_readfirstlane(TILES ? base + u : 0);  // the tile's chunk j is unit base + j * tiles
      w.chunk_len = len;
      w.s.row0 = __builtin_amdgcn_readfirstlane(s.row0);
      w.s.n = __builtin_amdgcn_readfirstlane(s.n);
      w.s.kv = __builtin_amdgcn_readfirstlane(s.kv);
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
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    return (uint32_t)f32_to_bf16_bits(lo) | ((uint32_t)f32_to_bf16_bits(hi) << 16);
  }
};
template <> struct Mat<f16_t> {
  static __device__ __forceinline__ f32x4_v run(u32x4_v a, u32x4_v b, f32x4_v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_v, a), __builtin_bit_cast(f16x8_v, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const f16_t a = (f16_t)lo, b = (f16_t)hi;
    uint16_t ua, ub;
    __builtin_memcpy(&ua, &a, 2);
    __builtin_memcpy(&ub, &b, 2);
    return (uint32_t)ua | ((uint32_t)ub << 16);
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
__device__ __forceinline__ void load_step(Step<T, HD> &f, const PagedArgs &p, int64_t head_at, int page_k, int page_v, int ks, int r, int g) {
  constexpr int E = Step<T, HD>::E, VE = Step<T, HD>::VE, VW = Step<T, HD>::VW;
  const int mask = (1 << p.page_shift) - 1;
  // an absent page's loads go to page 0, which exists; what they bring is not used
  const T *kr = (const T *)p.k + head_at + max(page_k, 0) * p.page_stride + ((ks + 8 * (r >> 2) + (r & 3)) & mask) * p.pos_stride + g * E;
#pragma unroll
  for (int kk = 0; kk < Step<T, HD>::KU; ++kk) {
    f.k0[kk] = *(const u32x4_v *)(kr + kk * 4 * E);
    f.k1[kk] = *(const u32x4_v *)(kr + 4 * p.pos_stride + kk * 4 * E);
  }
  const T *vr = (const T *)p.v + head_at + max(page_v, 0) * p.page_stride + ((ks + 8 * g) & mask) * p.pos_stride + r * VE;
#pragma unroll
  for (int i = 0; i < 8; ++i) __builtin_memcpy(f.v[i], __builtin_assume_aligned(vr + i * p.pos_stride, VW * 4 < 16 ? VW * 4 : 16), VW * 4);
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

// whether a word of cached values holds an infinity or a NaN
template <class T> __device__ __forceinline__ bool not_finite(uint32_t w) {
  constexpr uint32_t e = sizeof(T) == 4 ? 0x7f800000u : std::is_same<T, bf16_t>::value ? 0x7f80u : 0x7c00u;
  return (w & e) == e || (sizeof(T) == 2 && (w >> 16 & e) == e);
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

  const int64_t head_at = hk * a.p.head_stride;
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
    // Positions that some rows of the tile see and others do not: a weight of zero does not keep an infinity or a NaN out of the
    // product, so such positions leave it and are added below for the rows that see them.
    uint32_t odd = 0;  // bit 8g + i
    if (!whole && i0 != i1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bool any = false;
#pragma unroll
        for (int x = 0; x < St::VW; ++x) any |= not_finite<T>(cur.v[i][x]);
        const unsigned long long lanes = __ballot(any);
        if (lanes) {
#pragma unroll
          for (int x = 0; x < 4; ++x) odd |= (lanes >> (16 * x) & 0xffff) ? 1u << (8 * x + i) : 0u;
          const bool drop = odd >> (8 * g + i) & 1;
#pragma unroll
          for (int x = 0; x < St::VW; ++x) cur.v[i][x] = drop ? 0u : cur.v[i][x];
        }
      }
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
    if (odd) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        for (int x = 0; x < 4; ++x) {
          if (!(odd >> (8 * x + i) & 1)) continue;
          const int page = __shfl(pv, 16 * x, 64), key = ks + 8 * x + i;
          const T *src = (const T *)a.p.v + head_at + page * a.p.page_stride + (key & ((1 << a.p.page_shift) - 1)) * a.p.pos_stride + VE * 4 * g;
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            const float wt = __shfl(p[t][i], 16 * x + r, 64);
            if (wt == 0.f) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int ht = 0; ht < HT; ++ht) acc[t][ht][e] += wt * Conv<T>::ld(src, VE * e + ht);
          }
        }
      }
    }
    if (AHEAD) cur = nxt;
    else if (ks + 128 < k_end) load_step<T, HD>(cur, a.p, head_at, pk_n, pv_n, ks + 128, r, g);
    pv = pv_n;
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
struct Shape { int qt, R; int64_t tiles, units; bool join; };

// Query rows of a tile: as few as hold a sequence's, since a tile reads the cache once for all of its rows.
static Shape attend_shape(const spec_paged_cache *c, const spec_paged_batch *b, int n_q) {
  Shape s;
  const int64_t G = n_q / c->n_kv_heads, per = (int64_t)b->max_rows * G;
  s.qt = per <= 16 ? 1 : per <= 32 || c->dtype == SPEC_DTYPE_F32 ? 2 : 4;
  s.R = 16 * s.qt;
  s.tiles = std::min((int64_t)b->B * ((per + s.R - 1) / s.R), (int64_t)b->rows * G / s.R + b->B);
  s.join = b->max_len > PA_CHUNK_MIN;
  s.units = s.tiles + (s.join ? PA_SLOTS / c->n_kv_heads + 1 : 0);
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
  if (b->B == 0 || b->rows == 0) { s = Shape{1, 16, 0, 0, false}; return SPEC_OK; }
  s = attend_shape(c, b, n_q);
  if (s.units * c->n_kv_heads * 256 >= (int64_t)1 << 32 || s.tiles * c->n_kv_heads * s.qt * 256 >= (int64_t)1 << 32)
    return fail_noctx(SPEC_ERR_CAPACITY, "%s: %lld tiles of %d key heads are beyond one launch", who, (long long)s.units, c->n_kv_heads);
  return SPEC_OK;
}

template <class T, int HD, int QT>
static void attend_launch(const AttendArgs &a, const Shape &s, hipStream_t st) {
  hipLaunchKernelGGL((k_paged_attend<T, HD, QT>), dim3((unsigned)(s.units * a.p.n_kv_heads)), dim3(256), 0, st, a);
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
  a.slots = std::max(1, PA_SLOTS / cache->n_kv_heads);
  hipStream_t st = (hipStream_t)hip_stream;
  SPEC_DISPATCH_DTYPE(cache->dtype, T, {
    if (cache->head_dim == 64) {
      if (s.qt == 1) attend_launch<T, 64, 1>(a, s, st);
      else if (s.qt == 2) attend_launch<T, 64, 2>(a, s, st);
      else if constexpr (sizeof(T) == 2) attend_launch<T, 64, 4>(a, s, st);
    } else {
      if (s.qt == 1) attend_launch<T, 128, 1>(a, s, st);
      else if (s.qt == 2) attend_launch<T, 128, 2>(a, s, st);
      else if constexpr (sizeof(T) == 2) attend_launch<T, 128, 4>(a, s, st);
    }
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
