// Logits cut to what temperature, top-k, top-p and min-p leave of them, and a draw from that (include/spec.h states the rules).
//
// In the order of the tokens (larger logit first, then lower id) every rule keeps a first part, so a row's result is one border: the last token that is
// kept.  A token's place in the order is one number of 64 bits, its logit's bits turned round over its id.
//
// Whether a sum of weights reaches top_p of the total decides which token is the last, and it has to be the same whatever order the sum
// was taken in.  So weights are whole numbers of a unit and sums of them are exact.  One unit for all would leave the many small weights of a long tail few
// bits, and errors of equal weights add up (a tail of 151935 tokens of e^-25 in units of 2^-44: 89 tokens too few of 83266).  So a weight is a whole number of up to
// 2^shift times the unit of its octave, 2^-(shift + octave); the sum of a bin, which lies within an octave, is 64 bits, other sums are two of 64 bits in the last
// octave's unit.  Shift is 50 up to 4096 tokens, 44 with 151936.  The exponential is computed in 64 bits (a power of two times a polynomial of degree 10 on half an octave).
//
// Rows differ in what they ask for, and a row has more work than a compute unit does quickly, so that all but the search for the border
// is cut into pieces of rows:
//   k_row_maxima    the largest logit of every 16 tokens, and of every piece
//   k_row_masses    (rows with top-p over all tokens, or a large top-k) counts and sums of weights by bins of 1/64 octave of the weight
//   k_row_border    a workgroup a row: what may hold the border, listed in LDS and narrowed down 8 bits of its places at a time.  For a small top-k
//                   that are the tokens above the k-th largest of the 16s' maxima, else those up to the bin in which the count or the sum reaches
//                   its limit.  What the maxima rule out is not read.  Draws, where all that is kept is in the list.
//   k_row_finish    the result; logits that the maxima rule out are not read.  Sums of the kept weights by 256 tokens, for
//   k_row_draw      the other rows' draws.
// 64 x 4 rows of 50272 bf16 logits, each sequence with its own rules: 9 + 14 + 36 + 17 + 5 us of 80; 24 x 8 fp32 rows of 151936: 28 + 15 + 46 + 28 + 5 of
// 124; one row of 32000: greedy 14, top-k 26, top-p of flat logits 44.  The maxima and the result are at memory's rate (a copy's); the border is a chain of passes, 1.5 to 3 us
// each from the list, and of trips to L2 where it reads the row: a workgroup a row, those whose border lies among all tokens last.  A
// workgroup for all of a row took 113, 297 and 45: rows that need all their weights kept their CU while others had nothing to do.
// What cost most in LDS: additions that return a place in a list, all to one word (3000 of them 30 us), so that a wave counts its tokens first.
#include "spec_internal.h"
#include "device_utils.h"
#include <algorithm>
#include <cmath>

namespace spec {

typedef unsigned long long u64;

constexpr int TR_BINS = 2048, TR_PER_OCTAVE = 64, TR_OCTAVES = TR_BINS / TR_PER_OCTAVE;  // bins of weights; the last octave has all smaller ones
constexpr int TR_FINE = 256;   // parts that what is looked at is cut into
constexpr int TR_LAST = 128;   // tokens that are put in order at once
constexpr int TR_FEW = 1024;   // the largest top-k that goes by the maxima alone
constexpr int TR_PIECES = 64;  // of a row, for its maxima
// Pieces that a row with bins is cut into, at most: more fill the chip, but one workgroup reads the bins of all (16 KB each, some 0.3 us).  8, 12, 16 and 37
// pieces, us: one row of 151936 with top-p 54.9, 53.7, 53.7, 56.7; 8 of them 55.6, 54.7, 54.5, 60.8; 32 with a top-k of 30000 79.6, 83.4, 83.6, 86.7.
constexpr int TR_CUTS = 8;

// A whole number of up to 94 bits: its lower 36 bits and those above, which are added up apart (2^28 of each fit); `plain` carries.
struct Sum {
  static constexpr int LOW = 36;
  static constexpr u64 MASK = (1ull << LOW) - 1;
  u64 lo, hi;
  __device__ __forceinline__ Sum operator+(const Sum &o) const { return Sum{lo + o.lo, hi + o.hi}; }
  __device__ __forceinline__ Sum operator-(const Sum &o) const { return Sum{lo - o.lo, hi - o.hi}; }  // (only of a term that was added as it is: nothing is borrowed)
  __device__ __forceinline__ Sum plain() const { return Sum{lo & MASK, hi + (lo >> LOW)}; }
  __device__ __forceinline__ double about() const { return (double)hi * (MASK + 1) + (double)lo; }
  static __device__ __forceinline__ Sum whole(double v) {  // of one from 0 on, below 2^94
    const u64 hi = (u64)(v * (1. / (MASK + 1)));
    return Sum{(u64)(v - (double)hi * (MASK + 1)), hi};
  }
};
// as numbers; b: plain
__device__ __forceinline__ bool less(const Sum &a, const Sum &b) {
  const Sum x = a.plain();
  return x.hi < b.hi || (x.hi == b.hi && x.lo < b.lo);
}

// What is found out about a row: kept is a logit that is larger than last_z, or equal with an id up to last_id; x = (z - zero) / temp.
struct RowBorder {
  double c;  // log2(e) / temp
  float last_z, zero, temp;
  int last_id;
  int endless, drawn;
};

struct TruncateArgs {
  const void *logits;
  int64_t row_stride;
  int row0, q, V, shift;  // first row of the launch; rows of a sequence; bits of a weight
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
  float *out;
  const float *u;
  int32_t *tokens;
  // workspace
  float *piece_max, *max16;   // [rows][TR_PIECES], [rows][n16]
  RowBorder *border;          // [rows]
  Sum *sums;                  // [rows][stretches]
  u64 *masses;                // [rows][cuts][TR_BINS]
  uint32_t *counts;           // [rows][cuts][TR_BINS]
  int pieces, piece;          // pieces of a row and tokens of one (a multiple of 1024), for the maxima
  int cuts, cut, B;           // for the masses; sequences
  int n16, stretches;         // 16s and 256s of a row
};

// Four logits from token x on (a multiple of four) as they lie in memory, from within the row wherever x is.
template <class T, bool VEC> struct Quad {
  T v[4];
  __device__ __forceinline__ void load(const T *row, int x, int V) {
    if constexpr (VEC) {
      __builtin_memcpy(v, __builtin_assume_aligned(row + min(x, V - 4), 4 * sizeof(T)), 4 * sizeof(T));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = row[min(x + i, V - 1)];
    }
  }
  // NaN and what lies behind the row are -infinity
  __device__ __forceinline__ void numbers(int x, int V, float (&z)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = (VEC ? x : x + i) < V ? fmaxf(Conv<T>::ld(v, i), -INFINITY) : -INFINITY;
  }
};

// Logits as numbers that rise with them.
__device__ __forceinline__ uint32_t rank_of(float z) {
  const uint32_t b = __float_as_uint(z);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_rank(uint32_t up) { return __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up); }
// A token's place in the order.  (-0 and 0 are the same logit.)
__device__ __forceinline__ u64 place_of(float z, int id) { return (u64)~rank_of(z + 0.f) << 32 | (uint32_t)id; }
__device__ __forceinline__ float logit_of(u64 place) { return of_rank(~(uint32_t)(place >> 32)); }

// A row's weights: log2 of one, its bin and octave, and itself as a whole number.
struct Weights {
  double M, c;  // largest logit, log2(e) / temperature
  int shift;
  __device__ __forceinline__ double log2_of(float z) const { return fmax(((double)z - M) * c, -1100.); }  // (-infinity at any temperature as well)
  // y: a log2, up to 0.  Bins never fall as logits do.
  static __device__ __forceinline__ int bin(double y) { return min((int)(y * -TR_PER_OCTAVE), TR_BINS - 1); }
  static __device__ __forceinline__ int octave_of(int bin) { return (int)((uint32_t)bin / TR_PER_OCTAVE); }
  static __device__ __forceinline__ int octave(double y) { return min((int)-y, TR_OCTAVES - 1); }  // octave_of(bin(y))
  // in units of the octave's own
  __device__ __forceinline__ u64 number(double y, int octave) const {
    const double n = rint(y), f = y - n;
    // the Taylor series of 2^f: what is left out is below (ln 2 / 2)^11 / 11! = 2.2e-13 of it
    double p = 7.0549116208011233e-9;
    p = fma(p, f, 1.0178086009239699e-7);
    p = fma(p, f, 1.3215486790144309e-6);
    p = fma(p, f, 1.5252733804059840e-5);
    p = fma(p, f, 1.5403530393381609e-4);
    p = fma(p, f, 1.3333558146428443e-3);
    p = fma(p, f, 9.6181291076284772e-3);
    p = fma(p, f, 5.5504108664821580e-2);
    p = fma(p, f, 0.24022650695910071);
    p = fma(p, f, 0.69314718055994531);
    p = fma(p, f, 1.);
    const double v = ldexp(p, (int)n + octave + shift) + 4503599627370496.;  // 2^52: the sum's bits are the number, to nearest
    return __builtin_bit_cast(u64, v) & 0xfffffffffffffull;
  }
  // in units of the last octave's
  static __device__ __forceinline__ Sum in_last(u64 r, int octave) {
    return Sum{r << (TR_OCTAVES - 1 - octave) & Sum::MASK, r >> (Sum::LOW - TR_OCTAVES + 1 + octave)};
  }
  __device__ __forceinline__ Sum number(float z) const {
    const double y = log2_of(z);
    return in_last(number(y, octave(y)), octave(y));
  }
};

// What a row asks for, and what its weights are.
struct RowRules {
  float temp, p, floor_p;
  int k;
  bool by_k, by_p, few, dense;  // few: the border of top-k goes by the maxima; dense: bins are needed
  __device__ __forceinline__ RowRules(const TruncateArgs &a, int b) {
    temp = a.temperature ? a.temperature[b] : 1.f;
    const bool greedy = !(temp > 0.f);
    k = greedy ? 1 : a.top_k ? a.top_k[b] : 0;
    p = greedy || !a.top_p ? 1.f : a.top_p[b];
    floor_p = greedy || !a.min_p ? 0.f : a.min_p[b];
    if (greedy) temp = 1.f;
    by_k = k > 0 && k < a.V;
    by_p = p < 1.f && k != 1;
    few = by_k && k <= min(TR_FEW, a.n16 / 2);
    dense = k != 1 && !few && (by_k || by_p);
  }
};
struct RowScale {
  float top, zero;  // the largest logit; 0 where it is infinite: then infinite ones share the weight and the others have none, and 0 and -infinity stand for them
  bool endless;
  Weights wt;
  float per_unit;  // bins, about, to a logit
  __device__ __forceinline__ RowScale(const TruncateArgs &a, int row, float temp) {
    const int lane = threadIdx.x & 63;
    top = wave_max(a.piece_max[(int64_t)row * TR_PIECES + min(lane, a.pieces - 1)]);
    endless = top == INFINITY;
    zero = endless ? 0.f : top;
    wt = Weights{(double)zero, 1.4426950408889634074 / (double)temp, a.shift};
    per_unit = fminf((float)(wt.c * TR_PER_OCTAVE), 3e38f);
  }
  __device__ __forceinline__ float of(float z) const { return !endless ? z : z == INFINITY ? 0.f : -INFINITY; }
  __device__ __forceinline__ int bin(float z) const { return Weights::bin(wt.log2_of(z)); }
  // The largest logit up to `zero` in a bin from `first` on.  The wave tries 64 at a time.
  __device__ __forceinline__ float largest_from(int first) const {
    uint32_t is = rank_of(-INFINITY), past = rank_of(zero) + 1;  // it is from `is` on and before `past`
    while (past - is > 1) {
      const uint32_t part = (past - is + 63) / 64, at = is + ((threadIdx.x & 63) + 1) * part;
      is += part * (uint32_t)__popcll(__ballot(at < past && bin(of_rank(at)) >= first));
      past = min(past, is + part);
    }
    return of_rank(is);
  }
};

// What a workgroup of NT threads that looks for a border holds.
template <int NT> struct Truncate {
  static constexpr int WAVES = NT / 64, LIST = NT == 256 ? 1024 : 4096;
  Sum target, before, found_mass, wave_m[WAVES];  // target, before: of the search, here since a wave has no registers left for them
  u64 list[LIST], mass[TR_BINS], fine_lo[TR_FINE], fine_hi[TR_FINE], last_lo[TR_LAST], last_hi[TR_LAST], wave_u[2][WAVES], found_place;
  uint32_t cnt[TR_BINS], fine_cnt[TR_FINE], wave_c[WAVES], found_bin, found_cnt, found_n, listed, few;
  static constexpr int UNITS = TR_BINS / 2;  // sums of weights over stretches of the row, in the place of mass: lower limbs and upper ones
};

// Sums and maxima over the lanes of a wave up to each lane (so that the last one has that of all), without a trip through LDS.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t shifted(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ u64 shifted(u64 v) {
  return (u64)shifted<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | shifted<CTRL, ROWS>((uint32_t)v);
}
template <class V> __device__ __forceinline__ V sum_to_lane(V v) {
  v += shifted<0x111, 0xf>(v); v += shifted<0x112, 0xf>(v); v += shifted<0x114, 0xf>(v); v += shifted<0x118, 0xf>(v);
  v += shifted<0x142, 0xa>(v); v += shifted<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ Sum sum_to_lane(const Sum &v) { return Sum{sum_to_lane(v.lo), sum_to_lane(v.hi)}; }
__device__ __forceinline__ u64 max_to_lane(u64 v) {
  v = max(v, shifted<0x111, 0xf>(v)); v = max(v, shifted<0x112, 0xf>(v)); v = max(v, shifted<0x114, 0xf>(v)); v = max(v, shifted<0x118, 0xf>(v));
  v = max(v, shifted<0x142, 0xa>(v)); v = max(v, shifted<0x143, 0xc>(v));
  return v;
}

// The sums of counts and weights up to a thread's own, and of all.
template <int NT, class Sh>
__device__ __forceinline__ void scan(Sh &sh, uint32_t &c, Sum &m, uint32_t &all_c, Sum &all_m) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  c = sum_to_lane(c);
  m = sum_to_lane(m);
  __syncthreads();
  if (lane == 63) { sh.wave_c[wv] = c; sh.wave_m[wv] = m; }
  __syncthreads();
  all_c = 0; all_m = Sum{0, 0};
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i == wv) { c += all_c; m = m + all_m; }
    all_c += sh.wave_c[i]; all_m = all_m + sh.wave_m[i];
  }
}

// Among N bins of counts cnt[i] and sums masses(i, number of bins), the one in which sh.target is reached, by sum or by count; what lies before it goes on top
// of what is there in before_cnt and sh.before.  Leaves the bin and its count; false if no bin reaches it.
template <int NT, int N, class F>
__device__ __forceinline__ bool find_bin(Truncate<NT> &sh, const uint32_t *cnt, F masses, bool by_mass, uint32_t &before_cnt, int &bin, uint32_t &n) {
  constexpr int PER = (N + NT - 1) / NT;
  const int first = threadIdx.x * PER;
  const bool on = first < N;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) c += on ? cnt[first + i] : 0;
  Sum m = masses(on ? first : 0, std::integral_constant<int, PER>());
  if (!on) m = Sum{0, 0};
  uint32_t to_c = c, all_c;
  Sum to_m = m, all_m;
  __syncthreads();
  if (threadIdx.x == 0) sh.found_bin = ~0u;
  scan<NT>(sh, to_c, to_m, all_c, all_m);
  to_c += before_cnt; to_m = to_m + sh.before;
  const Sum target = sh.target;
  auto short_of = [&](uint32_t c, const Sum &m) { return by_mass ? less(m, target) : c < (uint32_t)target.lo; };
  Sum at = to_m - m;
  uint32_t at_c = to_c - c;
  if (!short_of(to_c, to_m) && short_of(at_c, at)) {
    // (sums only grow here: a bin taken off the sum of several may ask for a carry back)
#pragma unroll 1
    for (int i = first; i < first + PER; ++i) {
      const uint32_t next_c = at_c + cnt[i];
      const Sum next = at + masses(i, std::integral_constant<int, 1>());
      if (!short_of(next_c, next)) {
        sh.found_bin = i; sh.found_cnt = at_c; sh.found_mass = at; sh.found_n = cnt[i];
        break;
      }
      at_c = next_c; at = next;
    }
  }
  __syncthreads();
  bin = (int)sh.found_bin;
  if (bin < 0) return false;
  before_cnt = sh.found_cnt; n = sh.found_n;
  if (threadIdx.x == 0) sh.before = sh.found_mass;
  return true;
}

template <int CTRL> __device__ __forceinline__ float from_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

struct Kept {
  float last_z;
  int last_id;
  __device__ __forceinline__ bool operator()(float z, int id) const { return z > last_z || (z == last_z && id <= last_id); }
};

// What a draw needs of LDS (a workgroup that looked for a border has it).
template <int NT> struct DrawShared {
  Sum found_mass, wave_m[NT / 64];
  uint32_t wave_c[NT / 64], found_bin;
};

// The draw of a row: the first token with which the sum of the kept weights, in the order of ids, exceeds u times their total.  sums(i): of n stretches of
// per * 256 tokens.
template <class T, bool VEC, int NT, class Sh, class F>
__device__ __forceinline__ void draw_token(Sh &sh, const TruncateArgs &a, int row, const RowScale &sc, const Kept &kept, F sums, int n, int per) {
  const int lane = threadIdx.x & 63, each = (n + NT - 1) / NT, s0 = min(n, (int)threadIdx.x * each), s1 = min(n, s0 + each);
  const T *z_row = (const T *)a.logits + (int64_t)row * a.row_stride;
  Sum own{0, 0}, total;
  for (int s = s0; s < s1; ++s) own = own + sums(s);
  if (threadIdx.x == 0) { sh.found_bin = 0; sh.found_mass = Sum{0, 0}; }
  Sum to = own;
  uint32_t none = 0, no_c;
  scan<NT>(sh, none, to, no_c, total);
  // exceeded from `target` on
  total = total.plain();
  const double want = (double)a.u[row] * total.about();
  Sum target = want > 0. ? Sum::whole(fmin(want, total.about())) : Sum{0, 0};
  target = Sum{target.lo + 1, target.hi}.plain();
  if (less(total, target)) target = total;
  Sum at = to - own;
  if (less(at, target) && !less(to, target)) {
    for (int s = s0; s < s1; ++s) {
      const Sum next = at + sums(s);
      if (!less(next, target)) { sh.found_bin = s; sh.found_mass = at; break; }
      at = next;
    }
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  Sum before = sh.found_mass;
  for (int s = (int)sh.found_bin * per; s < min(a.stretches, ((int)sh.found_bin + 1) * per) && less(before, target); ++s) {
    const int x = 256 * s + 4 * lane;
    Quad<T, VEC> v;
    float z[4];
    v.load(z_row, x, a.V);
    v.numbers(x, a.V, z);
    Sum w[4], sum{0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      z[i] = sc.of(z[i]);
      w[i] = kept(z[i], x + i) ? sc.wt.number(z[i]) : Sum{0, 0};
      sum = sum + w[i];
    }
    const Sum up_to = sum_to_lane(sum);
    Sum c = before + up_to - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Sum next = c + w[i];
      if (less(c, target) && !less(next, target)) a.tokens[row] = x + i;
      c = next;
    }
    before = before + Sum{__shfl(up_to.lo, 63, 64), __shfl(up_to.hi, 63, 64)};
  }
}

// ------------------------------------------------------------------ pieces of rows
template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_row_maxima(TruncateArgs a) {
  __shared__ float sh[4];
  const int row = a.row0 + blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, V = a.V;
  const T *z_row = (const T *)a.logits + (int64_t)row * a.row_stride;
  float *max16 = a.max16 + (int64_t)row * a.n16;
  float top = -INFINITY;
  for (int x0 = piece * a.piece + 4 * threadIdx.x; x0 - 4 * (int)(threadIdx.x & 63) < min(V, (piece + 1) * a.piece); x0 += 4096) {  // (whole waves)
    Quad<T, VEC> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i].load(z_row, x0 + 1024 * i, V);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = x0 + 1024 * i;
      float z[4];
      v[i].numbers(x, V, z);
      float t = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
      t = fmaxf(t, from_lane<0xb1>(t));
      t = fmaxf(t, from_lane<0x4e>(t));
      top = fmaxf(top, t);
      if ((threadIdx.x & 3) == 0 && x < V) max16[x >> 4] = t;
    }
  }
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) a.piece_max[(int64_t)row * TR_PIECES + piece] = fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

// Which rows need bins is on the device.  With up to 64 sequences these rows share the pieces that there is room for, with more a row has its own.
struct Cuts {
  u64 dense;      // sequences that need bins
  int each, cut;  // pieces of a row, tokens of one
  __device__ __forceinline__ Cuts(const TruncateArgs &a) {
    dense = 0;
    each = a.cuts;
    if (a.B <= 64) {
      const int lane = threadIdx.x & 63;
      dense = __ballot(lane < a.B && RowRules(a, min(lane, a.B - 1)).dense);
      each = max(each, min(min(TR_CUTS, (a.V + 4095) / 4096), a.B * a.cuts / max(1, __popcll(dense))));
    }
    cut = ((a.V + each * 4096 - 1) / (each * 4096)) * 4096;
    each = (a.V + cut - 1) / cut;
  }
  // the first piece of a row
  __device__ __forceinline__ int64_t first(const TruncateArgs &a, int row) const {
    if (a.B > 64) return (int64_t)row * a.cuts;
    return (int64_t)(__popcll(dense & ((1ull << (row / a.q)) - 1)) * a.q + row % a.q) * each;
  }
};

template <class T, bool VEC>
__global__ __launch_bounds__(512) void k_row_masses(TruncateArgs a) {
  __shared__ u64 mass[TR_BINS];
  __shared__ uint32_t cnt[TR_BINS];
  const Cuts cuts(a);
  int row = a.row0 + blockIdx.x / cuts.each;
  const int cut = blockIdx.x % cuts.each, V = a.V;
  if (a.B <= 64) {  // (all rows are one launch's then)
    u64 left = cuts.dense;
    const int nth = row / a.q;
    if (nth >= __popcll(left)) return;
    for (int i = 0; i < nth; ++i) left &= left - 1;
    row = (__ffsll(left) - 1) * a.q + row % a.q;
  }
  const RowRules r(a, row / a.q);
  if (!r.dense) return;
  const RowScale sc(a, row, r.temp);
  if (sc.top == -INFINITY) return;
  const T *z_row = (const T *)a.logits + (int64_t)row * a.row_stride;
  for (int i = threadIdx.x; i < TR_BINS; i += 512) { mass[i] = 0; cnt[i] = 0; }
  __syncthreads();
  const int end = min(V, (cut + 1) * cuts.cut);
  for (int x0 = cut * cuts.cut + 4 * threadIdx.x; x0 < end; x0 += 8192) {
    Quad<T, VEC> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i].load(z_row, x0 + 2048 * i, V);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z[4];
      v[i].numbers(x0 + 2048 * i, end, z);
      u64 w[4];
      int at[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double y = sc.wt.log2_of(z[e] = sc.of(z[e]));
        at[e] = Weights::bin(y);
        w[e] = sc.wt.number(y, Weights::octave_of(at[e]));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (z[e] > -INFINITY) {
          atomicAdd(&mass[at[e]], w[e]);
          if (r.by_k) atomicAdd(&cnt[at[e]], 1u);
        }
      }
    }
  }
  __syncthreads();
  const int64_t at = (cuts.first(a, row) + cut) * TR_BINS;
  for (int i = threadIdx.x; i < TR_BINS; i += 512) {
    a.masses[at + i] = mass[i];
    if (r.by_k) a.counts[at + i] = cnt[i];
  }
}

// ------------------------------------------------------------------ the border
// (256 threads: three workgroups a CU, 600 x 2 rows of 8000 112 us, with two 127; rows that are not loaded in fours need registers for two.  512 threads: LDS has
// room for two workgroups, registers for one.)
template <class T, bool VEC, int NT>
__global__ __launch_bounds__(NT, NT == 256 && VEC ? 3 : 2) void k_row_border(TruncateArgs a) {
  typedef Truncate<NT> Sh;
  __shared__ Sh sh;
  const int row = a.row0 + blockIdx.x, lane = threadIdx.x & 63, wv = threadIdx.x >> 6, V = a.V;
  const T *z_row = (const T *)a.logits + (int64_t)row * a.row_stride;
  const float *max16 = a.max16 + (int64_t)row * a.n16;
  const RowRules r(a, row / a.q);
  const RowScale sc(a, row, r.temp);
  const Weights &wt = sc.wt;
  const int k = r.k;
  if (sc.top == -INFINITY) {
    if (threadIdx.x == 0) {
      a.border[row] = RowBorder{wt.c, INFINITY, 0.f, 1.f, -1, 0, 1};  // (INFINITY: of numbers that are not larger, none is kept)
      if (a.tokens) a.tokens[row] = 0;
    }
    return;
  }

  // the border: the place of the last token that top-k and top-p keep
  u64 border = ~0ull;
  bool from_list = false, all_listed = false;  // all_listed: the list has all that lies before the border as well
  if (k == 1) {
    // the lowest token of the largest logit, in the first 16 that have it
    if (threadIdx.x == 0) sh.few = ~0u;
    __syncthreads();
    uint32_t first = ~0u;
    for (int g = threadIdx.x; g < a.n16; g += 8 * NT) {
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = max16[min(g + i * NT, a.n16 - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (z[i] == sc.top) first = min(first, (uint32_t)min(g + i * NT, a.n16 - 1));
    }
    if (first != ~0u) atomicMin(&sh.few, first);
    __syncthreads();
    if (wv == 0) {
      const int id = 16 * (int)sh.few + (lane & 15);
      const u64 mask = __ballot(id < V && Conv<T>::ld(z_row, min(id, V - 1)) == sc.top);
      if (lane == 0) {
        sh.list[0] = place_of(sc.zero, 16 * (int)sh.few + (mask ? __ffsll(mask) - 1 : 0));
      }
    }
    __syncthreads();
    border = sh.list[0];
    if (a.tokens && threadIdx.x == 0) a.tokens[row] = (int)(uint32_t)border;
  } else if (r.by_k || r.by_p) {
    // What is looked at: the tokens of bins first .. last whose places lie in lo .. hi, n of them, of the row or of the list.  The border is the first of
    // them with which the count, or by_mass the sum, on top of bc or sh.before, reaches sh.target.  (n may be too small before they are listed or picked.)
    int first = 0, last = TR_BINS - 1;
    u64 lo = 0, hi = ~0ull;
    uint32_t n = 0, bc = 0, listing = 0;  // listing: tokens that a list takes, where there is room
    bool by_mass = false, searching = true;
    auto set = [&](Sum &x, const Sum &to) {  // (read behind the next barrier)
      if (threadIdx.x == 0) x = to;
    };
    set(sh.target, Sum{(u64)max(k, 1), 0});
    set(sh.before, Sum{0, 0});
    auto part_of = [&](const Sum &all) {
      const Sum total = all.plain(), part = Sum::whole(fmin(fmax(ceil((double)r.p * total.about()), 1.), total.about()));
      return less(part, total) ? part : total;
    };
    auto of_bins = [&](int i, auto N) {  // (of one octave)
      u64 m = 0;
#pragma unroll
      for (int j = 0; j < decltype(N)::value; ++j) m += sh.mass[i + j];
      return Weights::in_last(m, Weights::octave_of(i));
    };
    auto of_part = [&](int i, auto) { return Sum{sh.fine_lo[i], sh.fine_hi[i]}; };
    // The bin where the count or the sum reaches `target` is looked at; those before it are listed as well where there is room for all.
    auto look_at_bin = [&]() {
      bc = 0; lo = 0; hi = ~0ull;
      set(sh.before, Sum{0, 0});
      from_list = false;
      const bool there = find_bin<NT, TR_BINS>(sh, sh.cnt, of_bins, by_mass, bc, last, n);
      const bool with_front = bc + n <= Sh::LIST;
      first = with_front ? 0 : last;
      listing = with_front ? bc + n : n;
      return there;
    };
    if (r.few) {
      // The k-th largest of the 16s' maxima is no larger than the k-th of all, so that the tokens that are not in a bin behind its own, little
      // more than k, have the first k among them.  (Of fewer than k finite ones all are kept.)
      for (int i = threadIdx.x; i < TR_BINS; i += NT) { sh.cnt[i] = 0; sh.mass[i] = 0; }
      __syncthreads();
      for (int g = threadIdx.x; g < a.n16; g += 8 * NT) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = max16[min(g + i * NT, a.n16 - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = sc.of(z[i]);
          if (g + i * NT < a.n16 && y > -INFINITY) atomicAdd(&sh.cnt[sc.bin(y)], 1u);
        }
      }
      __syncthreads();
      if (!find_bin<NT, TR_BINS>(sh, sh.cnt, of_bins, false, bc, last, n)) last = TR_BINS - 1;
      bc = 0; n = listing = 0;
      set(sh.before, Sum{0, 0});
    } else {
      uint32_t c = 0, all_c;
      Sum m{0, 0}, all_m;
      constexpr int PER = (TR_BINS + NT - 1) / NT;
      const Cuts cuts(a);
      const int64_t at = cuts.first(a, row) * TR_BINS + threadIdx.x;
      u64 masses[PER] = {};
      uint32_t counts[PER] = {};
#pragma unroll 4
      for (int cut = 0; cut < cuts.each; ++cut)
#pragma unroll
        for (int i = 0; i < PER; ++i) masses[i] += a.masses[at + cut * TR_BINS + min(i * NT, TR_BINS - 1 - (int)threadIdx.x)];
      if (r.by_k)
        for (int cut = 0; cut < cuts.each; ++cut)
#pragma unroll
          for (int i = 0; i < PER; ++i) counts[i] += a.counts[at + cut * TR_BINS + min(i * NT, TR_BINS - 1 - (int)threadIdx.x)];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int of = threadIdx.x + i * NT;
        if (of >= TR_BINS) break;
        // A bin's weights are alike, so that its sum tells how many there are, a little high (the last one's, which may be small, aside).
        if (!r.by_k) counts[i] = masses[i] ? 1 + (uint32_t)(ldexpf((float)masses[i], -a.shift) * exp2f((of % TR_PER_OCTAVE + 1) * (1.01f / TR_PER_OCTAVE))) : 0;
        sh.mass[of] = masses[i]; sh.cnt[of] = counts[i];
        c += counts[i]; m = m + Weights::in_last(masses[i], Weights::octave_of(of));
      }
      scan<NT>(sh, c, m, all_c, all_m);
      by_mass = !(r.by_k && (uint32_t)k < all_c);
      if (by_mass) set(sh.target, part_of(all_m));
      searching = (r.by_p || !by_mass) && look_at_bin();
    }
    // One pass over what is looked at a turn, until it is few tokens: list it where there is room; else its bounds, and which of 256 parts between
    // them has the border.  (Eight bits of at most 64 every two turns, for two borders: the limit is never met.)
    enum { LIST, BOUNDS, PARTS, LAST };
    bool bounded = true;
    int drop = 0;
    u64 base = place_of(sc.zero, 0);
    // Parts from the first bin on: they need not end where the bins do.
    auto parts_to = [&](u64 end) {
      drop = max(0, 64 - __clzll(end - base) - 8);
      bounded = true;
    };
    auto parts_of_bins = [&]() {
      base = place_of(first == 0 ? sc.zero : sc.zero - (float)(first - 1) / sc.per_unit, 0);
      parts_to(max(base + 1, place_of(sc.zero - (float)(last + 2) / sc.per_unit, 0)));
    };
    parts_of_bins();
#pragma unroll 1
    for (int turn = 0; searching && turn < 48; ++turn) {
      const int mode = !from_list && listing <= Sh::LIST ? LIST : from_list && n <= TR_LAST ? LAST : bounded ? PARTS : BOUNDS;
      __syncthreads();
      if (threadIdx.x == 0) {
        if (mode == LIST) sh.listed = 0;
        sh.few = 0;
      }
      if (mode == PARTS)
        for (int i = threadIdx.x; i < TR_FINE; i += NT) { sh.fine_lo[i] = 0; sh.fine_hi[i] = 0; sh.fine_cnt[i] = 0; }
      __syncthreads();
      u64 least = ~0ull, most = 0;
      auto take = [&](u64 at, float z) {  // (lists and orders are below: a wave counts its tokens first, since a thousand additions to one word of LDS take 10 us)
        if (at < lo || at > hi) return;
        if (mode == BOUNDS) {
          least = min(least, at); most = max(most, at);
        } else {
          const int part = (int)min((u64)(TR_FINE - 1), (at - min(at, base)) >> drop);
          atomicAdd(&sh.fine_cnt[part], 1u);
          if (r.by_p) {
            const Sum w = wt.number(z);
            atomicAdd(&sh.fine_lo[part], w.lo);
            if (w.hi) atomicAdd(&sh.fine_hi[part], w.hi);
          }
        }
      };
      if (from_list) {
        const uint32_t listed = sh.listed;
#pragma unroll 1
        for (uint32_t i = threadIdx.x; i < listed; i += NT) {
          const u64 at = sh.list[i];
          if (mode == LAST) {
            const bool on = at >= lo && at <= hi;
            const u64 mask = __ballot(on);
            if (!mask) continue;
            const int leader = __ffsll(mask) - 1;
            uint32_t to = 0;
            if (lane == leader) to = atomicAdd(&sh.few, (uint32_t)__popcll(mask));
            to = __builtin_amdgcn_readlane(to, leader) + __popcll(mask & ((1ull << lane) - 1));
            if (on && to < TR_LAST) {
              const Sum w = wt.number(logit_of(at));
              sh.fine_lo[to] = at; sh.fine_lo[TR_LAST + to] = w.lo; sh.fine_hi[to] = w.hi;
            }
          } else {
            take(at, logit_of(at));
          }
        }
      } else {
        // A wave takes 4 x 64 of the 16s at a time and, of those whose maxima are not behind the last bin, a quad a lane.  What is taken of the quads
        // lies between two logits: one a little behind the last bin, whose tokens are no matter, and the largest of the first bin.  (With a bin worked out
        // for each token near it a row of 151936 whose border lies among all took 42 us, not 33.)
        const float d_last = last == TR_BINS - 1 ? INFINITY : (float)(last + 1) / sc.per_unit;
        const float low = sc.endless ? INFINITY : fmaxf(sc.zero - d_last - 1e-6f * (fabsf(sc.zero) + d_last), -3.4028235e38f);
        const float high = sc.endless ? INFINITY : first ? sc.largest_from(first) : sc.zero;
        const bool all = lo == 0 && hi == ~0ull;
#pragma unroll 1
        for (int g0 = 256 * wv; g0 < a.n16; g0 += 256 * Sh::WAVES) {
          int order[4], hits[4], rounds = 0;
          float z16[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) z16[i] = max16[min(g0 + 64 * i + lane, a.n16 - 1)];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool hit = g0 + 64 * i + lane < a.n16 && z16[i] >= low && z16[i] > -INFINITY;
            const u64 mask = __ballot(hit);
            const int before = __popcll(mask & ((1ull << lane) - 1));
            hits[i] = __popcll(mask);
            order[i] = __builtin_amdgcn_ds_permute(4 * (hit ? before : hits[i] + lane - before), lane);  // those first
            rounds = max(rounds, (hits[i] + 15) / 16);
          }
          Quad<T, VEC> ahead[4];
          int ahead_x[4];
          auto load = [&](int round) {
            const int nth = 16 * round + (lane >> 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int g = g0 + 64 * i + __builtin_amdgcn_ds_bpermute(4 * nth, order[i]);
              ahead_x[i] = nth < hits[i] ? 16 * g + 4 * (lane & 3) : V;  // (V: none)
              ahead[i].load(z_row, ahead_x[i], V);
            }
          };
          load(0);
#pragma unroll 1
          for (int round = 0; round < rounds; ++round) {
            Quad<T, VEC> v[4];
            int x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = ahead[i]; x[i] = ahead_x[i]; }
            load(round + 1);  // (behind the last one: none)
            float z[4][4];
            int in[4], own = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              in[i] = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                z[i][e] = Conv<T>::ld(v[i].v, e);
                in[i] |= (z[i][e] >= low && z[i][e] <= high && (VEC || x[i] + e < V)) << e;
              }
              if (x[i] >= V) in[i] = 0;
              if (sc.endless) {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[i][e] = sc.of(z[i][e]);
              }
              if (!all && in[i]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const u64 at = place_of(z[i][e], x[i] + e);
                  in[i] &= ~((at < lo || at > hi) << e);
                }
              }
              own += __popc(in[i]);
            }
            if (mode == LIST) {
              if (!__any(own)) continue;
              const uint32_t upto = sum_to_lane((uint32_t)own), whole = __builtin_amdgcn_readlane(upto, 63);
              uint32_t to = 0;
              if (lane == 63) to = atomicAdd(&sh.listed, whole);
              to = __builtin_amdgcn_readlane(to, 63) + upto - own;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (!in[i]) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (in[i] >> e & 1) {
                    if (to < Sh::LIST) sh.list[to] = place_of(z[i][e], x[i] + e);
                    ++to;
                  }
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
#pragma unroll 1
                for (int e = 0; e < 4; ++e)
                  if (in[i] >> e & 1) {
                    const float y = e == 0 ? z[i][0] : e == 1 ? z[i][1] : e == 2 ? z[i][2] : z[i][3];
                    take(place_of(y, x[i] + e), y);
                  }
              }
            }
          }
        }
      }
      __syncthreads();
      if (mode == LIST) {
        listing = sh.listed;
        from_list = listing <= Sh::LIST;
        all_listed = lo == 0 && first == 0;
        const bool in_front = !r.few && all_listed && last > 0;  // tokens that bc and sh.before count have been listed with the bin's own
        if (!in_front || !from_list) n = listing;
        if (in_front) {
          lo = base = place_of(sc.largest_from(last), 0);
          parts_to(max(base + 1, place_of(sc.zero - (float)(last + 2) / sc.per_unit, 0)));
        }
        if (r.few && !by_mass && n <= (uint32_t)k && from_list && all_listed) {  // fewer finite ones than asked for, or just as many
          set(sh.target, Sum{n, 0});
          searching = n > 0;
        }
      } else if (mode == BOUNDS) {
        least = ~max_to_lane(~least);
        most = max_to_lane(most);
        if (lane == 63) { sh.wave_u[0][wv] = least; sh.wave_u[1][wv] = most; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) { least = min(least, sh.wave_u[0][i]); most = max(most, sh.wave_u[1][i]); }
        lo = base = least;
        hi = most;
        parts_to(hi);
      } else if (mode == PARTS) {
        int part;
        searching = find_bin<NT, TR_FINE>(sh, sh.fine_cnt, of_part, by_mass, bc, part, n);
        const u64 begin = base + ((u64)part << drop);
        if (part > 0) lo = max(lo, begin);
        if (part < TR_FINE - 1) hi = min(hi, begin + ((1ull << drop) - 1));
        if (!from_list) listing = n;
        bounded = false;
      } else if (sh.few > TR_LAST) {  // (a bin's number of tokens is known about)
        n = sh.few;
      } else {
        // Few tokens: four threads each, which add up those of a quarter of them that come up to it.  (Their sums go where none of the others' is read.)
        if (threadIdx.x == 0) sh.found_place = ~0ull;
        auto of_token = [&](int i) { return Sum{sh.fine_lo[TR_LAST + i], sh.fine_hi[i]}; };
        auto up_to_token = [&](int i) { return Sum{sh.last_lo[i], sh.last_hi[i]}; };
        for (int i = threadIdx.x; i < TR_LAST; i += NT) { sh.fine_cnt[i] = bc; sh.last_lo[i] = sh.before.lo; sh.last_hi[i] = sh.before.hi; }
        __syncthreads();
        const int some = (int)min(sh.few, (uint32_t)TR_LAST);
        for (int i = threadIdx.x; i < 4 * TR_LAST; i += NT) {
          const int of = i % TR_LAST, j0 = i / TR_LAST * (TR_LAST / 4);
          if (of >= some || j0 >= some) continue;
          const u64 own = sh.fine_lo[of];
          uint32_t c = 0;
          u64 m_lo = 0, m_hi = 0;
#pragma unroll 1
          for (int j = j0; j < min(some, j0 + TR_LAST / 4); j += 8) {
            u64 other[8], lo8[8], hi8[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) { other[e] = sh.fine_lo[j + e]; lo8[e] = sh.fine_lo[TR_LAST + j + e]; hi8[e] = sh.fine_hi[j + e]; }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const bool upto = j + e < some && other[e] <= own;
              c += upto;
              m_lo += upto ? lo8[e] : 0;
              m_hi += upto ? hi8[e] : 0;
            }
          }
          atomicAdd(&sh.fine_cnt[of], c);
          atomicAdd(&sh.last_lo[of], m_lo);
          atomicAdd(&sh.last_hi[of], m_hi);
        }
        __syncthreads();
        if ((int)threadIdx.x < some) {
          const Sum m = up_to_token(threadIdx.x), target = sh.target;
          if (by_mass ? !less(m, target) && less(m - of_token(threadIdx.x), target) : sh.fine_cnt[threadIdx.x] == (uint32_t)target.lo) {
            sh.found_place = sh.fine_lo[threadIdx.x]; sh.found_mass = m;
          }
        }
        __syncthreads();
        border = sh.found_place;
        searching = false;
        if (r.by_p && !by_mass && border != ~0ull) {  // of the first k their sum, and its part, which is reached among them at the latest
          by_mass = true;
          const Sum target = part_of(sh.found_mass);
          const bool among = less(sh.before, target);  // these tokens, whose sums are there
          __syncthreads();  // (all have read the first border and what lies before it)
          set(sh.target, target);
          if (among) {
            if ((int)threadIdx.x < some) {
              const Sum m = up_to_token(threadIdx.x);
              if (!less(m, target) && less(m - of_token(threadIdx.x), target)) sh.found_place = sh.fine_lo[threadIdx.x];
            }
            __syncthreads();
            border = sh.found_place;
          } else if (r.few) {
            lo = 0; hi = border; bc = 0;
            set(sh.before, Sum{0, 0});
            n = listing = (uint32_t)k;
            from_list = from_list && all_listed;
            base = place_of(sc.zero, 0);
            parts_to(border);
            searching = true;
          } else {  // (the bins need not know of the first k)
            searching = look_at_bin();
            parts_of_bins();
          }
        }
      }
    }
  }

  // The border as a logit and, among equal ones, a token: kept is what is larger, or equal and not behind it.
  float last_z = border == ~0ull ? -INFINITY : logit_of(border);
  int last_id = border == ~0ull ? -1 : (int)(uint32_t)border;
  if (r.floor_p > 0.f && wt.c > 0.) {
    // min-p as a border: the lowest logit whose weight is enough, which is next to what the logarithm gives, and the largest logit at most
    const double least = log2((double)fminf(r.floor_p, 1.f));
    float z = nextafterf(nextafterf((float)(wt.M + least / wt.c), -INFINITY), -INFINITY);
    for (int i = 0; i < 6 && !(wt.log2_of(z) >= least); ++i) z = nextafterf(z, INFINITY);
    z = fminf(z, sc.zero);
    if (z > last_z) { last_z = nextafterf(z, -INFINITY); last_id = -1; }
  }
  const bool draw = a.tokens && border != ~0ull && from_list && all_listed;
  if (threadIdx.x == 0) a.border[row] = RowBorder{wt.c, last_z, sc.zero, r.temp, last_id, sc.endless, draw || k == 1};
  if (!draw) return;
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * Sh::UNITS; i += NT) sh.mass[i] = 0;
  __syncthreads();
  const Kept kept{last_z, last_id};
  const int per = (a.stretches + Sh::UNITS - 1) / Sh::UNITS;
  for (uint32_t i = threadIdx.x; i < sh.listed; i += NT) {
    const u64 at = sh.list[i];
    const int id = (int)(uint32_t)at;
    if (kept(logit_of(at), id)) {
      const Sum w = wt.number(logit_of(at));
      atomicAdd(&sh.mass[(id >> 8) / per], w.lo);
      if (w.hi) atomicAdd(&sh.mass[Sh::UNITS + (id >> 8) / per], w.hi);
    }
  }
  __syncthreads();
  draw_token<T, VEC, NT>(sh, a, row, sc, kept, [&](int i) { return Sum{sh.mass[i], sh.mass[Sh::UNITS + i]}; }, Sh::UNITS, per);
}

// ------------------------------------------------------------------ the result
template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_row_finish(TruncateArgs a, int pieces, bool write, bool add) {
  const int row = a.row0 + blockIdx.x / pieces, piece = blockIdx.x % pieces, V = a.V, lane = threadIdx.x & 63;
  const T *z_row = (const T *)a.logits + (int64_t)row * a.row_stride;
  const float *max16 = a.max16 + (int64_t)row * a.n16;
  float *out = write ? a.out + (int64_t)row * V : nullptr;
  const RowBorder rb = a.border[row];
  const Kept kept{rb.last_z, rb.last_id};
  const Weights wt{(double)rb.zero, rb.c, a.shift};
  const double per_temp = 1. / (double)rb.temp;
  add = add && !rb.drawn;
  if (!write && !add) return;
  const int x0 = piece * 4096 + 4 * threadIdx.x;
  float top[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) top[i] = max16[min(x0 + 1024 * i, V - 1) >> 4];
  Quad<T, VEC> v[4];
  bool some[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float t = !rb.endless ? top[i] : top[i] == INFINITY ? 0.f : -INFINITY;
    some[i] = t >= rb.last_z && t > -INFINITY;
    if (some[i]) v[i].load(z_row, x0 + 1024 * i, V);
  }
  // (A loop: unrolled, this kernel is 15 KB of instructions, not 4.)
#pragma unroll 1
  for (int x = x0; x < x0 + 4096 && x - 4 * lane < V; x += 1024) {
    float y[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    Sum w{0, 0};
    if (some[0]) {
      float z[4];
      v[0].numbers(x, V, z);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (rb.endless) z[e] = z[e] == INFINITY ? 0.f : -INFINITY;
        if (kept(z[e], x + e)) {
          y[e] = (float)(((double)z[e] - rb.zero) * per_temp);  // (rounded once; the difference alone may leave fp32)
          if (add) w = w + wt.number(z[e]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) { v[i] = v[i + 1]; some[i] = some[i + 1]; }
    if (add) {
      if (__any((w.lo | w.hi) != 0)) w = sum_to_lane(w);
      if (lane == 63) a.sums[(int64_t)row * a.stretches + (x >> 8)] = w;
    }
    if (write) {
      if constexpr (VEC) {
        if (x < V) *(float4 *)(out + x) = make_float4(y[0], y[1], y[2], y[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (x + e < V) out[x + e] = y[e];
      }
    }
  }
}

template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_row_draw(TruncateArgs a) {
  __shared__ DrawShared<256> sh;
  const int row = a.row0 + blockIdx.x;
  const RowBorder rb = a.border[row];
  if (rb.drawn) return;
  const RowScale sc(a, row, rb.temp);
  const Sum *sums = a.sums + (int64_t)row * a.stretches;
  draw_token<T, VEC, 256>(sh, a, row, sc, Kept{rb.last_z, rb.last_id}, [&](int i) { return sums[i]; }, a.stretches, 1);
}

}  // namespace spec

using namespace spec;

static int truncate_check(const char *who, int32_t B, int32_t s, int32_t vocab) {
  if (B < 0 || s < 0 || vocab < 1) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: B=%d s=%d vocab=%d", who, B, s, vocab);
  if (s > 15 || B > 65535 || vocab > (1 << 28)) return fail_noctx(SPEC_ERR_CAPACITY, "%s: at most s = 15, B = 65535, vocab = 2^28", who);
  return SPEC_OK;
}

// The pieces of a call's rows and where the workspace has what; -> its bytes.
static size_t truncate_layout(TruncateArgs &a, int64_t rows, void *workspace) {
  const int V = a.V;
  auto up = [](int64_t n, int64_t to) { return (n + to - 1) / to; };
  a.piece = (int)(up(up(V, 4096), TR_PIECES) * 4096);
  a.pieces = (int)up(V, a.piece);
  // bins cost 24 KB a piece, written and read again: as many pieces as it takes to fill the chip, of 4096 tokens at least
  a.cuts = (int)std::max<int64_t>(1, std::min({up(V, 4096), up(1024, std::max<int64_t>(1, rows)), (int64_t)TR_CUTS}));
  a.cuts = (int)up(V, up(V, (int64_t)a.cuts * 4096) * 4096);
  a.n16 = (int)up(V, 16);
  a.stretches = (int)up(V, 256);
  size_t at = 0;
  auto take = [&](auto *&p, size_t n) {
    p = (std::remove_reference_t<decltype(p)>)((char *)workspace + at);
    at += (n * sizeof(*p) + 255) / 256 * 256;
  };
  take(a.piece_max, rows * TR_PIECES);
  take(a.max16, rows * a.n16);
  take(a.border, rows);
  take(a.sums, rows * a.stretches);
  take(a.masses, rows * a.cuts * TR_BINS);
  take(a.counts, rows * a.cuts * TR_BINS);
  return at;
}

extern "C" int spec_truncate_logits_workspace_bytes(int32_t B, int32_t s, int32_t vocab, size_t *bytes) {
  const char *who = "spec_truncate_logits_workspace_bytes";
  if (!bytes) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: bytes is null", who);
  const int rc = truncate_check(who, B, s, vocab);
  if (rc) return rc;
  TruncateArgs a{};
  a.V = vocab;
  *bytes = truncate_layout(a, (int64_t)B * (s + 1), nullptr);
  return SPEC_OK;
}

extern "C" int spec_truncate_logits(void *hip_stream, const void *d_logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t s, int32_t vocab,
                                    const spec_sampling_rules *rules, const float *d_uniforms, void *d_workspace, size_t workspace_bytes,
                                    float *d_out, int32_t *d_tokens) {
  const char *who = "spec_truncate_logits";
  const int rc = truncate_check(who, B, s, vocab);
  if (rc) return rc;
  if (dtype < SPEC_DTYPE_F32 || dtype > SPEC_DTYPE_F16) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (row_stride < vocab) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: row_stride is shorter than a row of %d", who, vocab);
  if (!rules) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: rules are null", who);
  if (B == 0) return SPEC_OK;
  if (!d_logits || (!d_out && !d_tokens)) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: null pointer", who);
  if (d_tokens && !d_uniforms) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: tokens need d_uniforms", who);
  if (((uintptr_t)d_logits % dtype_bytes(dtype)) || ((uintptr_t)d_out & 3)) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: misaligned pointer", who);
  const bool in_place = (const void *)d_out == d_logits;
  if (in_place && (dtype != SPEC_DTYPE_F32 || row_stride != vocab))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: in place only for fp32 rows without padding", who);
  int bits = 0;
  while (bits < 28 && (1 << bits) < vocab) ++bits;
  const int rows = B * (s + 1);
  TruncateArgs a{d_logits, row_stride, 0, s + 1, vocab, std::min(50, 62 - bits), rules->d_temperature, rules->d_top_k, rules->d_top_p, rules->d_min_p,
                 d_out, d_uniforms, d_tokens};
  a.B = B;
  const size_t need = truncate_layout(a, rows, d_workspace);
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || workspace_bytes < need)
    return fail_noctx(SPEC_ERR_WORKSPACE, "%s: workspace null, not 256-byte aligned, or smaller than %zu bytes", who, need);
  hipStream_t st = (hipStream_t)hip_stream;
  const int fours = (vocab + 4095) / 4096;
  const int most = std::max(1, ((1 << 24) - 1) / std::max(fours, 4));  // rows of a launch: a grid holds less than 2^32 threads
  SPEC_DISPATCH_DTYPE(dtype, T, {
    const bool vec = vocab % 4 == 0 && row_stride % 4 == 0 && (uintptr_t)d_logits % (4 * sizeof(T)) == 0 && (uintptr_t)d_out % 16 == 0;
    auto launch = [&](auto VEC_) {
      constexpr bool VEC = decltype(VEC_)::value;
      auto each = [&](auto f) {  // launches of up to `most` rows
        for (a.row0 = 0; a.row0 < rows; a.row0 += most) f((unsigned)std::min(most, rows - a.row0));
        a.row0 = 0;
      };
      const bool first = d_out && !(in_place && d_tokens);  // (in place the draw reads the row before it goes)
      each([&](unsigned n) { hipLaunchKernelGGL((k_row_maxima<T, VEC>), dim3(n * a.pieces), dim3(256), 0, st, a); });
      if (rules->d_top_p || rules->d_top_k) {
        if (B <= 64) hipLaunchKernelGGL((k_row_masses<T, VEC>), dim3(rows * a.cuts), dim3(512), 0, st, a);
        else each([&](unsigned n) { hipLaunchKernelGGL((k_row_masses<T, VEC>), dim3(n * a.cuts), dim3(512), 0, st, a); });
      }
      each([&](unsigned n) {
        if (vocab > 8192) hipLaunchKernelGGL((k_row_border<T, VEC, 512>), dim3(n), dim3(512), 0, st, a);
        else hipLaunchKernelGGL((k_row_border<T, VEC, 256>), dim3(n), dim3(256), 0, st, a);
      });
      each([&](unsigned n) { hipLaunchKernelGGL((k_row_finish<T, VEC>), dim3(n * fours), dim3(256), 0, st, a, fours, first, d_tokens != nullptr); });
      if (d_tokens) each([&](unsigned n) { hipLaunchKernelGGL((k_row_draw<T, VEC>), dim3(n), dim3(256), 0, st, a); });
      if (d_out && !first) each([&](unsigned n) { hipLaunchKernelGGL((k_row_finish<T, VEC>), dim3(n * fours), dim3(256), 0, st, a, fours, true, false); });
    };
    if (vec) launch(std::true_type());
    else launch(std::false_type());
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
