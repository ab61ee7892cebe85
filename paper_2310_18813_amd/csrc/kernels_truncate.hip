// Logits cut to what temperature, top-k, top-p and min-p leave of them, and a draw from that (include/spec.h states the rules).
//
// In the order of the tokens (larger logit first, then lower id) every rule keeps a first part, so a row's result is one border: the last token that is
// kept.  A token's place in the order is one number of 64 bits, its logit's bits turned round over its id.
//
// Whether a sum of weights reaches top_p of the total decides which token is the last, and it has to be the same whatever order the sum
// was taken in.  So weights are whole numbers, e^x times a power of two to nearest, and sums of them are exact: 2^50 for
// a weight of 1 up to 4096 tokens, 2^44 with 151936.  Their exponential is computed in 64 bits (a power of two times a polynomial of degree 10 on half an octave).
//
// A workgroup takes a row.  Passes: the largest logit; counts and sums of weights by bins of 1/64 octave of the weight, in LDS; the tokens of
// the bin with the border, listed in LDS and narrowed down; the result.  Only where a bin has more tokens than the list does narrowing go over the row.
#include "spec_internal.h"
#include "device_utils.h"
#include <algorithm>
#include <cmath>

namespace spec {

typedef unsigned long long u64;

constexpr int TR_BINS = 2048, TR_LIST = 4096, TR_FINE = 256, TR_SEGS = 256;

struct TruncateArgs {
  const void *logits;
  int64_t row_stride;
  int q, V, shift;  // rows of a sequence; a weight of 1 is 2^shift
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
  float *out;
  const float *u;
  int32_t *tokens;
};

// Four logits from token x on (a multiple of four); NaN and what lies behind the row are -infinity.
template <class T, bool VEC>
__device__ __forceinline__ void row4(const T *row, int x, int V, float (&z)[4]) {
  if constexpr (VEC) {
    T v[4];
    const int at = min(x, V - 4);
    __builtin_memcpy(v, __builtin_assume_aligned(row + at, 4 * sizeof(T)), 4 * sizeof(T));
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = x < V ? fmaxf(Conv<T>::ld(v, i), -INFINITY) : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = Conv<T>::ld(row, min(x + i, V - 1));
      z[i] = x + i < V ? fmaxf(v, -INFINITY) : -INFINITY;
    }
  }
}

// A token's place in the order.  (-0 and 0 are the same logit.)
__device__ __forceinline__ u64 place_of(float z, int id) {
  const uint32_t b = __float_as_uint(z + 0.f);
  const uint32_t up = b & 0x80000000u ? ~b : b | 0x80000000u;  // rises with the logit
  return (u64)~up << 32 | (uint32_t)id;
}
__device__ __forceinline__ float logit_of(u64 place) {
  const uint32_t up = ~(uint32_t)(place >> 32);
  return __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
}

// A row's weights: log2 of one, its bin, and itself as a whole number.
struct Weights {
  double M, c;  // largest logit, log2(e) / temperature
  int shift;
  __device__ __forceinline__ double log2_of(float z) const { return fmax(((double)z - M) * c, -1100.); }  // (-infinity at any temperature as well)
  __device__ __forceinline__ int bin(double y) const { return min(TR_BINS - 1, (int)(y * -64.)); }
  __device__ __forceinline__ u64 number(double y) const {
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
    const double v = ldexp(p, (int)n + shift) + 4503599627370496.;  // 2^52: the sum's bits are the number, to nearest
    return __builtin_bit_cast(u64, v) & 0xfffffffffffffull;
  }
};

template <int NT> struct TruncateShared {
  u64 list[TR_LIST], mass[TR_BINS], fine_mass[TR_FINE], seg[TR_SEGS], wave_u[2][NT / 64], found_mass, found_place;
  uint32_t cnt[TR_BINS], fine_cnt[TR_FINE], wave_c[NT / 64], found_bin, found_cnt, found_n, listed;
};

__device__ __forceinline__ u64 wave_sum(u64 v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The sums of counts and weights up to a thread's own, and of all.  (Reads back sh.wave_*: two barriers.)
template <int NT>
__device__ __forceinline__ void scan(TruncateShared<NT> &sh, uint32_t &c, u64 &m, uint32_t &all_c, u64 &all_m) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t uc = __shfl_up(c, o, 64);
    const u64 um = __shfl_up(m, o, 64);
    if (lane >= o) { c += uc; m += um; }
  }
  __syncthreads();
  if (lane == 63) { sh.wave_c[wv] = c; sh.wave_u[0][wv] = m; }
  __syncthreads();
  all_c = 0; all_m = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i == wv) { c += all_c; m += all_m; }
    all_c += sh.wave_c[i]; all_m += sh.wave_u[0][i];
  }
}

// Among N bins of counts and sums, the one in which `target` is reached, by sum or by count; what lies before it goes on top of what
// is there in before_*.  Leaves the bin and its count; false if no bin reaches it.
template <int NT, int N>
__device__ __forceinline__ bool find_bin(TruncateShared<NT> &sh, const uint32_t *cnt, const u64 *mass, bool by_mass, u64 target, uint32_t &before_cnt,
                                         u64 &before_mass, int &bin, uint32_t &n) {
  constexpr int PER = N / NT > 0 ? N / NT : 1;
  const int first = threadIdx.x * PER;
  uint32_t c[PER];
  u64 m[PER];
  uint32_t sc = 0;
  u64 sm = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool on = first + i < N;
    c[i] = on ? cnt[first + i] : 0; m[i] = on ? mass[first + i] : 0;
    sc += c[i]; sm += m[i];
  }
  uint32_t to_c = sc, all_c;
  u64 to_m = sm, all_m;
  if (threadIdx.x == 0) sh.found_bin = ~0u;
  scan<NT>(sh, to_c, to_m, all_c, all_m);
  to_c += before_cnt - sc; to_m += before_mass - sm;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const u64 was = by_mass ? to_m : to_c, is = was + (by_mass ? m[i] : c[i]);
    if (was < target && is >= target) {
      sh.found_bin = first + i; sh.found_cnt = to_c; sh.found_mass = to_m; sh.found_n = c[i];
    }
    to_c += c[i]; to_m += m[i];
  }
  __syncthreads();
  bin = (int)sh.found_bin;
  if (bin < 0) return false;
  before_cnt = sh.found_cnt; before_mass = sh.found_mass; n = sh.found_n;
  return true;
}

template <class T, bool VEC, int NT>
__global__ __launch_bounds__(NT) void k_truncate_logits(TruncateArgs a) {
  __shared__ TruncateShared<NT> sh;
  const int row = blockIdx.x, b = row / a.q, lane = threadIdx.x & 63, wv = threadIdx.x >> 6, V = a.V;
  const T *z_row = (const T *)a.logits + (int64_t)row * a.row_stride;
  float *out = a.out ? a.out + (int64_t)row * V : nullptr;
  float temp = a.temperature ? a.temperature[b] : 1.f;
  const bool greedy = !(temp > 0.f);
  int k = greedy ? 1 : a.top_k ? a.top_k[b] : 0;
  const float p = greedy || !a.top_p ? 1.f : a.top_p[b];
  float floor_p = greedy || !a.min_p ? 0.f : a.min_p[b];
  if (greedy) temp = 1.f;

  // the largest logit and its lowest token
  u64 best = ~0ull;
  for (int x = 4 * threadIdx.x; x < V; x += 4 * NT) {
    float z[4];
    row4<T, VEC>(z_row, x, V, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) best = min(best, place_of(z[i], x + i));
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) best = min(best, (u64)__shfl_xor(best, o, 64));
  if (lane == 0) sh.wave_u[0][wv] = best;
  for (int i = threadIdx.x; i < TR_BINS; i += NT) { sh.mass[i] = 0; sh.cnt[i] = 0; }
  for (int i = threadIdx.x; i < TR_SEGS; i += NT) sh.seg[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) best = min(best, sh.wave_u[0][i]);
  const float top = logit_of(best);
  if (top == -INFINITY) {
    if (out)
      for (int x = threadIdx.x; x < V; x += NT) out[x] = -INFINITY;
    if (threadIdx.x == 0 && a.tokens) a.tokens[row] = 0;
    return;
  }
  // Where the largest is infinite, infinite ones share the weight and the others have none: 0 and -infinity instead of them.
  const bool endless = top == INFINITY;
  const Weights wt{endless ? 0. : (double)top, 1.4426950408889634074 / (double)temp, a.shift};
  auto fetch = [&](int x, float (&z)[4]) {
    row4<T, VEC>(z_row, x, V, z);
    if (endless) {
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = z[i] == INFINITY ? 0.f : -INFINITY;
    }
  };

  // the border: the place of the last token that top-k and top-p keep
  u64 border = ~0ull;
  if (k == 1) {
    border = endless ? place_of(0.f, (int)(uint32_t)best) : best;
  } else if ((k > 0 && k < V) || p < 1.f) {
    for (int x = 4 * threadIdx.x; x < V; x += 4 * NT) {
      float z[4];
      fetch(x, z);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (z[i] == -INFINITY) continue;
        const double y = wt.log2_of(z[i]);
        const int bin = wt.bin(y);
        atomicAdd(&sh.cnt[bin], 1u);
        atomicAdd(&sh.mass[bin], wt.number(y));
      }
    }
    __syncthreads();
    uint32_t all_c = 0;
    u64 all_m = 0;
    {
      uint32_t c = 0;
      u64 m = 0;
      for (int i = threadIdx.x; i < TR_BINS; i += NT) { c += sh.cnt[i]; m += sh.mass[i]; }
      scan<NT>(sh, c, m, all_c, all_m);
    }

    // The first token, among those of bin `of`, with which count or sum reaches `target` -> its place; before_*: in front of the bin, then up to
    // and with the token.
    auto resolve = [&](int of, uint32_t n, bool by_mass, u64 target, uint32_t &before_cnt, u64 &before_mass) {
      u64 lo = 0, hi = ~0ull;
      bool listed = false;
      auto each = [&](auto f) {
        if (listed) {
          for (uint32_t i = threadIdx.x; i < min(sh.listed, (uint32_t)TR_LIST); i += NT) {
            const u64 at = sh.list[i];
            if (at >= lo && at <= hi) f(at);
          }
        } else {
          for (int x = 4 * threadIdx.x; x < V; x += 4 * NT) {
            float z[4];
            fetch(x, z);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (z[i] == -INFINITY || wt.bin(wt.log2_of(z[i])) != of) continue;
              const u64 at = place_of(z[i], x + i);
              if (at >= lo && at <= hi) f(at);
            }
          }
        }
      };
      // (every turn takes 8 of at most 64 bits)
      for (int turn = 0; turn < 10; ++turn) {
        if (!listed && n <= TR_LIST) {
          __syncthreads();
          if (threadIdx.x == 0) sh.listed = 0;
          __syncthreads();
          each([&](u64 at) { const uint32_t i = atomicAdd(&sh.listed, 1u); if (i < TR_LIST) sh.list[i] = at; });
          __syncthreads();
          listed = true;
        }
        if (n <= 64) break;
        u64 least = ~0ull, most = 0;
        each([&](u64 at) { least = min(least, at); most = max(most, at); });
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) { least = min(least, (u64)__shfl_xor(least, o, 64)); most = max(most, (u64)__shfl_xor(most, o, 64)); }
        __syncthreads();
        if (lane == 0) { sh.wave_u[0][wv] = least; sh.wave_u[1][wv] = most; }
        for (int i = threadIdx.x; i < TR_FINE; i += NT) { sh.fine_mass[i] = 0; sh.fine_cnt[i] = 0; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) { least = min(least, sh.wave_u[0][i]); most = max(most, sh.wave_u[1][i]); }
        lo = least; hi = most;
        const int bits = 64 - __clzll(hi - lo), sh_r = max(0, bits - 8);
        each([&](u64 at) {
          const int bin = (int)((at - lo) >> sh_r);
          atomicAdd(&sh.fine_cnt[bin], 1u);
          atomicAdd(&sh.fine_mass[bin], wt.number(wt.log2_of(logit_of(at))));
        });
        __syncthreads();
        int bin;
        if (!find_bin<NT, TR_FINE>(sh, sh.fine_cnt, sh.fine_mass, by_mass, target, before_cnt, before_mass, bin, n)) break;
        lo += (u64)bin << sh_r;
        hi = lo + min(hi - lo, (1ull << sh_r) - 1);
      }
      __syncthreads();
      if (threadIdx.x == 0) { sh.found_place = ~0ull; sh.found_cnt = before_cnt; sh.found_mass = before_mass; }
      // 64 tokens at most: a lane each, which adds up those up to its own
      if (wv == 0) {
        u64 mine = ~0ull;
        const uint32_t listed_n = min(sh.listed, (uint32_t)TR_LIST);
        n = min(n, 64u);
        uint32_t have = 0;
        for (uint32_t i = 0; i < listed_n; i += 64) {  // (all of them, of which n lie in the interval)
          const u64 at = i + lane < listed_n ? sh.list[i + lane] : ~0ull;
          const u64 in = __ballot(at >= lo && at <= hi && i + lane < listed_n);
          const uint32_t rank = have + __popcll(in & ((1ull << lane) - 1));
          if (in >> lane & 1 && rank < 64) sh.fine_mass[rank] = at;
          have += __popcll(in);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < (int)n) mine = sh.fine_mass[lane];
        const u64 w = lane < (int)n ? wt.number(wt.log2_of(logit_of(mine))) : 0;
        uint32_t c = before_cnt;
        u64 m = before_mass;
        for (int j = 0; j < (int)n; ++j) {
          const u64 other = __shfl(mine, j, 64), ow = __shfl(w, j, 64);
          if (other <= mine) { ++c; m += ow; }
        }
        const u64 is = by_mass ? m : c, was = is - (by_mass ? w : 1);
        if (lane < (int)n && was < target && is >= target) { sh.found_place = mine; sh.found_cnt = c; sh.found_mass = m; }
      }
      __syncthreads();
      before_cnt = sh.found_cnt; before_mass = sh.found_mass;
      return sh.found_place;
    };

    int bin;
    uint32_t n, bc = 0;
    u64 bm = 0;
    if (k > 0 && (uint32_t)k < all_c) {
      find_bin<NT, TR_BINS>(sh, sh.cnt, sh.mass, false, (u64)k, bc, bm, bin, n);
      border = resolve(bin, n, false, (u64)k, bc, bm);
      all_m = bm;
    }
    if (p < 1.f) {
      const u64 target = max((u64)1, min(all_m, (u64)ceil(fmax((double)p, 0.) * (double)all_m)));
      bc = 0; bm = 0;
      __syncthreads();
      find_bin<NT, TR_BINS>(sh, sh.cnt, sh.mass, true, target, bc, bm, bin, n);
      border = resolve(bin, n, true, target, bc, bm);
    }
  }
  // as a logit and, among equal ones, a token
  const float last_z = border == ~0ull ? -INFINITY : logit_of(border);
  const int last_id = border == ~0ull ? -1 : (int)(uint32_t)border;
  const bool floored = floor_p > 0.f;
  const double least = floored ? log2((double)fminf(floor_p, 1.f)) : 0.;
  auto kept = [&](float z, int id) { return (z > last_z || (z == last_z && id <= last_id)) && (!floored || wt.log2_of(z) >= least); };
  const float zero = endless ? 0.f : top;

  const int steps = (V + 4 * NT - 1) / (4 * NT), per = (steps + TR_SEGS - 1) / TR_SEGS;
  const bool in_place = (const void *)out == (const void *)z_row;
  if (a.tokens) __syncthreads();
  auto finish = [&](bool write, bool add) {
    for (int step = 0; step < steps; ++step) {
      const int x = 4 * (step * NT + threadIdx.x);
      float z[4];
      fetch(x, z);
      u64 w = 0;
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = -INFINITY;
        if (kept(z[i], x + i)) {
          if (add) w += wt.number(wt.log2_of(z[i]));
          y[i] = (z[i] - zero) / temp;
        }
      }
      if (write) {
        if constexpr (VEC) {
          if (x < V) *(float4 *)(out + x) = make_float4(y[0], y[1], y[2], y[3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (x + i < V) out[x + i] = y[i];
        }
      }
      if (add && __any(w != 0)) {
        w = wave_sum(w);
        if (lane == 0) atomicAdd(&sh.seg[step / per], w);
      }
    }
  };
  if (out && !(in_place && a.tokens)) finish(true, a.tokens != nullptr);
  else finish(false, true);
  if (!a.tokens) return;

  // the draw: the first token with which the sum of the kept weights, in the order of ids, exceeds u times their total
  __syncthreads();
  u64 total = 0;
  for (int i = 0; i < TR_SEGS; ++i) total += sh.seg[i];
  const double want = (double)a.u[row] * (double)total;
  const u64 target = want > 0. ? min(total - 1, (u64)want) : 0;  // exceeded from target + 1 on
  u64 before = 0;
  int seg = 0;
  while (seg < TR_SEGS - 1 && before + sh.seg[seg] <= target) before += sh.seg[seg++];
  for (int step = seg * per; step < min(steps, seg * per + per); ++step) {
    const int x = 4 * (step * NT + threadIdx.x);
    float z[4];
    fetch(x, z);
    u64 w[4], to = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = kept(z[i], x + i) ? wt.number(wt.log2_of(z[i])) : 0;
      to += w[i];
    }
    uint32_t c = 0, all_c;
    u64 all, at = before - to;
    scan<NT>(sh, c, to, all_c, all);
    at += to;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at <= target && at + w[i] > target) a.tokens[row] = x + i;
      at += w[i];
    }
    before += all;
    if (before > target) break;
  }
  if (out && in_place) {
    __syncthreads();
    finish(true, false);
  }
}

}  // namespace spec

using namespace spec;

static int truncate_check(const char *who, int32_t B, int32_t s, int32_t vocab) {
  if (B < 0 || s < 0 || vocab < 1) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: B=%d s=%d vocab=%d", who, B, s, vocab);
  if (s > 15 || B > 65535 || vocab > (1 << 28)) return fail_noctx(SPEC_ERR_CAPACITY, "%s: at most s = 15, B = 65535, vocab = 2^28", who);
  return SPEC_OK;
}

extern "C" int spec_truncate_logits_workspace_bytes(int32_t B, int32_t s, int32_t vocab, size_t *bytes) {
  const char *who = "spec_truncate_logits_workspace_bytes";
  if (!bytes) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: bytes is null", who);
  const int rc = truncate_check(who, B, s, vocab);
  if (rc) return rc;
  *bytes = 0;
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
  if ((const void *)d_out == d_logits && (dtype != SPEC_DTYPE_F32 || row_stride != vocab))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: in place only for fp32 rows without padding", who);
  int bits = 0;
  while (bits < 28 && (1 << bits) < vocab) ++bits;
  TruncateArgs a{d_logits, row_stride, s + 1, vocab, std::min(50, 62 - bits), rules->d_temperature, rules->d_top_k, rules->d_top_p, rules->d_min_p,
                 d_out, d_uniforms, d_tokens};
  SPEC_DISPATCH_DTYPE(dtype, T, {
    const bool vec = vocab % 4 == 0 && row_stride % 4 == 0 && (uintptr_t)d_logits % (4 * sizeof(T)) == 0 && (uintptr_t)d_out % 16 == 0;
    if (vocab > 8192)
      hipLaunchKernelGGL((vec ? k_truncate_logits<T, true, 1024> : k_truncate_logits<T, false, 1024>), dim3(B * (s + 1)), dim3(1024), 0,
                         (hipStream_t)hip_stream, a);
    else
      hipLaunchKernelGGL((vec ? k_truncate_logits<T, true, 256> : k_truncate_logits<T, false, 256>), dim3(B * (s + 1)), dim3(256), 0,
                         (hipStream_t)hip_stream, a);
  });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
