// Penalties for repeated tokens, biases and a grammar's mask on logits, in front of the acceptance rules (include/spec.h states them).
//
// A workgroup takes a piece of the vocabulary of one sequence and all its rows of logits, or a group of them.  It counts the sequence's
// tokens that fall into the piece in LDS -- the whole list is read for every piece, from L2 after the first, which is why pieces are as
// long as still fill the chip -- and then streams its rows through: a thread keeps the counts and biases of four tokens in registers for
// all rows.  Counts are integers, so their order is no matter; a token of the proposals carries a mark, and only marked tokens compare with
// them row by row.  Nothing is kept between calls: a rejected proposal needs no taking back.
//
// Bound by memory: 4 or 2 bytes read and 4 written a logit, an eighth of a byte of mask.
#include "spec_internal.h"
#include "device_utils.h"
#include <algorithm>

// fp32 as the rules are stated, operation by operation
#pragma clang fp contract(off)

namespace spec {

constexpr uint32_t LR_PROMPT = 1u << 31, LR_PROPOSED = 1u << 30, LR_COUNT = LR_PROPOSED - 1;
constexpr int LR_ROWS = 4;  // rows whose loads are in flight together

struct LogitArgs {
  const void *logits;
  int64_t row_stride;
  int s, V, piece, rows;  // tokens of a piece, rows of a workgroup
  spec_logit_rules r;
  const int32_t *t;
  int t_stride;
  float *out;
};

template <class T, bool VEC>
__device__ __forceinline__ void load4(const T *row, int x, int V, float (&z)[4]) {
  if constexpr (VEC) {
    T v[4];
    __builtin_memcpy(v, __builtin_assume_aligned(row + x, 4 * sizeof(T)), 4 * sizeof(T));
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = Conv<T>::ld(v, i);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = Conv<T>::ld(row, min(x + i, V - 1));
  }
}

template <class T, bool VEC, int NT>
__global__ __launch_bounds__(NT) void k_process_logits(LogitArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lr_smem[];
  uint32_t *cnt = lr_smem, *last = lr_smem + a.piece;  // counts; 1 + index of a token's bias (only with biases)
  const int b = blockIdx.y, c0 = blockIdx.x * a.piece, j0 = blockIdx.z * a.rows, j1 = min(j0 + a.rows, a.s + 1);
  const int words = a.r.n_bias ? 2 * a.piece : a.piece;
  for (int x = 4 * threadIdx.x; x < words; x += 4 * NT) *(uint4 *)(lr_smem + x) = make_uint4(0, 0, 0, 0);
  __syncthreads();
  if (a.r.d_tokens) {
    const int n = (int)min((int64_t)max(a.r.d_len[b], 0), a.r.tokens_stride), prompt = a.r.d_prompt_len ? a.r.d_prompt_len[b] : 0;
    const int32_t *tok = a.r.d_tokens + b * a.r.tokens_stride;
    for (int i0 = threadIdx.x; i0 < n; i0 += 8 * NT) {
      int v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = tok[min(i0 + NT * k, n - 1)];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + NT * k, x = v[k] - c0;
        if (i < n && v[k] >= c0 && v[k] < a.V && x < a.piece) {
          if (i < prompt) atomicOr(&cnt[x], LR_PROMPT);
          else atomicAdd(&cnt[x], 1u);
        }
      }
    }
  }
  const int32_t *t = a.t ? a.t + (int64_t)b * a.t_stride : nullptr;
  if (t && (int)threadIdx.x < a.s) {
    const int v = t[threadIdx.x];
    if (v >= c0 && v < a.V && v - c0 < a.piece) atomicOr(&cnt[v - c0], LR_PROPOSED);
  }
  const float *bias = a.r.d_bias + (int64_t)b * a.r.n_bias;
  for (int i = threadIdx.x; i < a.r.n_bias; i += NT) {
    const int v = a.r.d_bias_ids[(int64_t)b * a.r.n_bias + i];
    if (v >= c0 && v < a.V && v - c0 < a.piece) atomicMax(&last[v - c0], (uint32_t)(i + 1));
  }
  __syncthreads();

  const float rep = a.r.d_repetition ? a.r.d_repetition[b] : 1.f;
  const float freq = a.r.d_frequency ? a.r.d_frequency[b] : 0.f, pres = a.r.d_presence ? a.r.d_presence[b] : 0.f;
  const T *rows = (const T *)a.logits + (int64_t)b * (a.s + 1) * a.row_stride;
  float *out = a.out + (int64_t)b * (a.s + 1) * a.V;
  const int mask_words = (a.V + 31) / 32;
  for (int x = 4 * threadIdx.x; x < a.piece && c0 + x < a.V; x += 4 * NT) {
    const uint4 w4 = *(const uint4 *)(cnt + x);
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    const bool seen = (w4.x | w4.y | w4.z | w4.w) != 0;
    float add[4] = {0.f, 0.f, 0.f, 0.f};
    bool biased = false;
    if (a.r.n_bias) {
      const uint4 l4 = *(const uint4 *)(last + x);
      biased = (l4.x | l4.y | l4.z | l4.w) != 0;
      if (l4.x) add[0] = bias[l4.x - 1];
      if (l4.y) add[1] = bias[l4.y - 1];
      if (l4.z) add[2] = bias[l4.z - 1];
      if (l4.w) add[3] = bias[l4.w - 1];
    }
    for (int jb = j0; jb < j1; jb += LR_ROWS) {
      float z[LR_ROWS][4];
      uint32_t allowed[LR_ROWS];
#pragma unroll
      for (int k = 0; k < LR_ROWS; ++k) {
        const int j = min(jb + k, j1 - 1);
        load4<T, VEC>(rows + j * a.row_stride, c0 + x, a.V, z[k]);
        allowed[k] = 15;
        if (a.r.d_mask)
          allowed[k] = a.r.d_mask[((int64_t)b * a.r.mask_rows + (a.r.mask_rows == 1 ? 0 : j)) * mask_words + (c0 + x) / 32] >> ((c0 + x) & 31);
      }
#pragma unroll
      for (int k = 0; k < LR_ROWS; ++k) {
        const int j = jb + k;
        if (j >= j1) break;
        if (seen) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (!w[i]) continue;
            int c = w[i] & LR_COUNT;
            if (w[i] & LR_PROPOSED)
              for (int e = 0; e < j; ++e) c += t[e] == c0 + x + i;
            if (c || (w[i] & LR_PROMPT)) z[k][i] = z[k][i] > 0.f ? z[k][i] / rep : z[k][i] * rep;
            z[k][i] = z[k][i] - (freq * (float)c + (c ? pres : 0.f));
          }
        }
        if (biased) {
#pragma unroll
          for (int i = 0; i < 4; ++i) z[k][i] = z[k][i] + add[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) z[k][i] = allowed[k] >> i & 1 ? z[k][i] : -INFINITY;
        float *dst = out + (int64_t)j * a.V + c0 + x;
        if constexpr (VEC) {
          *(float4 *)dst = make_float4(z[k][0], z[k][1], z[k][2], z[k][3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c0 + x + i < a.V) dst[i] = z[k][i];
        }
      }
    }
  }
}

int logit_rules_check(const char *who, const spec_logit_rules *r, int s) {
  if (!r) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: rules are null", who);
  if (r->n_bias < 0 || (r->n_bias > 0 && (!r->d_bias_ids || !r->d_bias))) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: n_bias=%d without its arrays", who, r->n_bias);
  if (r->n_bias > 4096) return fail_noctx(SPEC_ERR_CAPACITY, "%s: at most 4096 biases a sequence", who);
  if (r->d_mask && r->mask_rows != 1 && r->mask_rows != s + 1)
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: mask_rows=%d is neither 1 nor %d", who, r->mask_rows, s + 1);
  return SPEC_OK;
}

void launch_process_logits(const void *logits, int dtype, int64_t row_stride, int B, int s, int V, const spec_logit_rules &r,
                           const int32_t *t, int t_stride, float *out, hipStream_t st) {
  LogitArgs a{logits, row_stride, s, V, 1024, s + 1, r, t, t_stride, out};
  if (!r.d_mask) a.r.mask_rows = 1;
  // Every workgroup of a sequence goes through all its tokens.  Where these can be many (their number is on the device: the list's room tells), workgroups of
  // 512 threads and pieces that leave 1024 workgroups; else 256 threads and 2048 workgroups.  us with 512 and with 256 threads, bf16: 64 rows of 50272
  // logits with 16000 tokens each 19.3 and 23.9, with 4000 13.2 and 14.6, with 1000 12.1 and 11.5; 24 x 8 rows of 151936 with 16000 46.5 and 48.4, with
  // 500 38.4 and 37.9.  It does not pay where few sequences have several long rows: 8 x 4 rows of 151936 with 16000 17.3 and 15.0.  Pieces half as long:
  // 24 x 8 fp32 rows of 151936 with up to 16000 tokens 53 -> 58.
  const bool many = r.d_tokens && r.tokens_stride > 4096;
  const int longest = r.n_bias ? 4096 : 8192, enough = many ? 1024 : 2048;
  while (a.piece < longest && (int64_t)B * ((V + 2 * a.piece - 1) / (2 * a.piece)) >= enough) a.piece *= 2;
  const int pieces = (V + a.piece - 1) / a.piece;
  while (a.rows > LR_ROWS && (int64_t)B * pieces * ((s + a.rows) / a.rows) < 512) a.rows = (a.rows + 1) / 2;
  const size_t lds = (size_t)a.piece * (r.n_bias ? 8 : 4);
  const dim3 grid(pieces, B, (s + a.rows) / a.rows);
  SPEC_DISPATCH_DTYPE(dtype, T, {
    const bool vec = V % 4 == 0 && row_stride % 4 == 0 && (uintptr_t)logits % (4 * sizeof(T)) == 0 && (uintptr_t)out % 16 == 0;
    if (many)
      hipLaunchKernelGGL((vec ? k_process_logits<T, true, 512> : k_process_logits<T, false, 512>), grid, dim3(512), lds, st, a);
    else
      hipLaunchKernelGGL((vec ? k_process_logits<T, true, 256> : k_process_logits<T, false, 256>), grid, dim3(256), lds, st, a);
  });
}

}  // namespace spec

using namespace spec;

extern "C" int spec_process_logits(void *hip_stream, const void *d_logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t s,
                                   int32_t vocab, const spec_logit_rules *rules, const int32_t *d_proposals, float *d_out) {
  const char *who = "spec_process_logits";
  if (B < 0 || s < 0 || vocab < 1) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: B=%d s=%d vocab=%d", who, B, s, vocab);
  if (s > 15 || B > 65535 || vocab > (1 << 28)) return fail_noctx(SPEC_ERR_CAPACITY, "%s: at most s = 15, B = 65535, vocab = 2^28", who);
  if (dtype < SPEC_DTYPE_F32 || dtype > SPEC_DTYPE_F16) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (row_stride < vocab) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: row_stride is shorter than a row of %d", who, vocab);
  const int rc = logit_rules_check(who, rules, s);
  if (rc) return rc;
  if (rules->d_tokens && (!rules->d_len || rules->tokens_stride < 1))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: d_tokens needs d_len and tokens_stride", who);
  if (rules->tokens_stride >= 1 << 30) return fail_noctx(SPEC_ERR_CAPACITY, "%s: at most 2^30 tokens a sequence", who);
  if (B == 0) return SPEC_OK;
  if (!d_logits || !d_out) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: null pointer", who);
  if (((uintptr_t)d_logits % dtype_bytes(dtype)) || ((uintptr_t)d_out & 3)) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: misaligned pointer", who);
  if ((const void *)d_out == d_logits && (dtype != SPEC_DTYPE_F32 || row_stride != vocab))
    return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: in place only for fp32 rows without padding", who);
  // a grid holds less than 2^32 threads
  const int64_t per = ((int64_t)vocab + 1023) / 1024 * 4 * 512;
  const int most = (int)std::max<int64_t>(1, (((int64_t)1 << 32) - 1) / per);
  for (int b0 = 0; b0 < B; b0 += most) {
    const int nb = std::min(most, B - b0);
    spec_logit_rules r = *rules;
    auto on = [&](auto *&p, int64_t n) { if (p) p += (int64_t)b0 * n; };
    on(r.d_tokens, r.tokens_stride); on(r.d_prompt_len, 1); on(r.d_len, 1);
    on(r.d_repetition, 1); on(r.d_frequency, 1); on(r.d_presence, 1);
    on(r.d_bias_ids, r.n_bias); on(r.d_bias, r.n_bias); on(r.d_mask, (int64_t)r.mask_rows * ((vocab + 31) / 32));
    launch_process_logits((const unsigned char *)d_logits + (int64_t)b0 * (s + 1) * row_stride * dtype_bytes(dtype), dtype, row_stride, nb, s, vocab, r,
                          d_proposals ? d_proposals + (int64_t)b0 * s : nullptr, s, d_out + (int64_t)b0 * (s + 1) * vocab, (hipStream_t)hip_stream);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
