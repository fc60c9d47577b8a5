// Rules on logits (atspeed_logit_rules): penalties for tokens that occurred,
// biases, temperature and grammar masks, one pass over the logits.
#include <algorithm>

#include "common.h"
#include "paged.h"

namespace atspeed {

// One workgroup per row and chunk of 256 * VEC * ITER columns.  Occurrences are
// counted in LDS by integer atomics (their order does not matter) from the history
// and the row's path; then every logit is read once and written once.  The logits and
// the row's state are requested before the request is searched, so a short row costs
// the chain lengths -> tokens -> output and a long one streams.  61 rows x 32 users of
// 1,024 fp32 columns: 5.1 us; 128 rows of 33,024 bf16 columns with 2,048 tokens of
// history (26 MB): 11.3, 2.3 TB/s, and 9.2 with one token.
constexpr int kRuleThreads = 256;

template <class T, int VEC> struct LogitVec;
template <> struct LogitVec<float, 4> {
  static __device__ __forceinline__ void ld(const float* p, float (&x)[4]) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  }
};
template <> struct LogitVec<bf16_t, 4> {
  static __device__ __forceinline__ void ld(const bf16_t* p, float (&x)[4]) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(v.x << 16);
    x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16);
    x[3] = __uint_as_float(v.y & 0xffff0000u);
  }
};
template <class T> struct LogitVec<T, 1> {
  static __device__ __forceinline__ void ld(const T* p, float (&x)[1]) { x[0] = St<T>::ld(p); }
};

// Divisions by a request's numbers are products with their reciprocals: half a step more
// of rounding, and a third of the instructions of an exact one per logit (128 rows of
// 33,024 columns: 10.7 us; divided 12.5, and the same with the product corrected by its
// residual).  In two factors, the second a power of two, so that the reciprocals of all
// positive numbers fit.
struct Reciprocal {
  float inv, scale;
  __device__ __forceinline__ explicit Reciprocal(float b) : scale(b < 0x1p-100f ? 0x1p64f : b > 0x1p100f ? 0x1p-64f : 1.f) {
    inv = 1.f / (b * scale);
  }
  __device__ __forceinline__ float times(float y) const { return y * inv * scale; }
};

template <class T, int VEC, int ITER>
__global__ void __launch_bounds__(kRuleThreads) logit_rules_kernel(atspeed_logit_rules_args a, int chunks, float lowest) {
  constexpr int CH = kRuleThreads * VEC * ITER;
  __shared__ int count[CH];
  __shared__ int s_user;
  const int tid = threadIdx.x, r = blockIdx.x / chunks, c0 = (blockIdx.x % chunks) * CH;
  const T* in = static_cast<const T*>(a.logits) + (int64_t)r * a.logits_stride;
  float x[ITER][VEC];
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const int c = c0 + (k * kRuleThreads + tid) * VEC;
    if (c + VEC <= a.n_cols) {
      LogitVec<T, VEC>::ld(in + c, x[k]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[k][e] = c + e < a.n_cols ? St<T>::ld(in + c + e) : 0.f;
    }
  }
  int state = a.allowed && !a.state_by_request ? a.state[r] : -1;
  const int orow = a.out_row ? a.out_row[r] : r;
  const bool counting = (a.repetition || a.frequency || a.presence) && (a.history || a.node_token);
  if (counting)
#pragma unroll
    for (int k = 0; k < CH / kRuleThreads; ++k) count[k * kRuleThreads + tid] = 0;
  if (tid == 0) s_user = -1;
  __syncthreads();
  for (int b = tid; b < a.B; b += kRuleThreads)
    if (a.row_off[b] <= r && r < a.row_off[b + 1]) s_user = b;
  __syncthreads();
  const int b = s_user;
  if (b < 0 || (a.out_row && (unsigned)orow >= (unsigned)a.n_out_rows)) return;

  if (counting) {
    auto see = [&](int token) {
      const long long col = (long long)token - a.token_base - c0;
      if (col >= 0 && col < CH) atomicAdd(&count[col], 1);
    };
    if (a.history) {
      const int n = min(a.hist_len[b], a.max_hist);
      const int* h = a.history + (int64_t)b * a.max_hist;
      for (int i = tid; i < n; i += kRuleThreads) see(h[i]);
    }
    if (a.node_token) {
      const int* tok = a.node_token + (int64_t)b * a.max_nodes;
      const uint64_t* m = a.mask ? a.mask + (int64_t)r * a.mask_words : nullptr;
      const int n = (int)min((int64_t)a.max_nodes, m ? (int64_t)a.mask_words * 64 : r - (int64_t)a.row_off[b] + 1);
      for (int j = tid; j < n; j += kRuleThreads)
        if (!m || ((m[j >> 6] >> (j & 63)) & 1)) see(tok[j]);
    }
    __syncthreads();
  }
  const float rep = a.repetition ? a.repetition[b] : 1.f;
  const Reciprocal rep_inv(rep), temp_inv(a.temperature ? a.temperature[b] : 1.f);
  const float freq = a.frequency ? a.frequency[b] : 0.f;
  const float pres = a.presence ? a.presence[b] : 0.f;
  const int bi = a.bias ? (a.bias_index ? a.bias_index[b] : 0) : -1;
  const float* bias = bi >= 0 && bi < a.n_bias ? a.bias + (int64_t)bi * a.bias_stride : nullptr;
  if (a.allowed && a.state_by_request) state = a.state[b];
  const bool masked = state >= 0;
  const uint32_t* allowed = masked && state < a.n_states ? a.allowed + (int64_t)state * ((a.n_cols + 31) / 32) : nullptr;
  float* out = a.out + (int64_t)orow * a.out_stride;
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const int off = (k * kRuleThreads + tid) * VEC, c = c0 + off;
    if (c >= a.n_cols) continue;
    const bool whole = c + VEC <= a.n_cols;
    float bv[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) bv[e] = 0.f;
    if (bias) {
      if (whole) {
        LogitVec<float, VEC>::ld(bias + c, bv);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (c + e < a.n_cols) bv[e] = bias[c + e];
      }
    }
    const uint32_t word = masked ? (allowed ? allowed[c >> 5] >> (c & 31) : 0u) : ~0u;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float y = x[k][e];
      const int n = counting ? count[off + e] : 0;
      if (n > 0) {
        if (a.repetition) y = y > 0.f ? rep_inv.times(y) : y * rep;
        y -= freq * (float)n + pres;
      }
      if (bias) y += bv[e];
      y = temp_inv.times(y);
      if (y < lowest) y = lowest;
      x[k][e] = (word >> e) & 1u ? y : a.mask_value;
    }
    if (VEC == 4 && whole) {
      *reinterpret_cast<f32x4_t*>(out + c) = f32x4_t{x[k][0], x[k][VEC > 1 ? 1 : 0], x[k][VEC > 2 ? 2 : 0], x[k][VEC > 3 ? 3 : 0]};
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c + e < a.n_cols) out[c + e] = x[k][e];
    }
  }
}

template <class T, int VEC, int ITER>
static atspeed_status launch_rules(const atspeed_logit_rules_args& a, float lowest, hipStream_t st) {
  const int ch = kRuleThreads * VEC * ITER, chunks = (a.n_cols + ch - 1) / ch;
  const long long n = (long long)chunks * a.n_rows;
  if (n > kMaxGroups) return fail(ATSPEED_E_SHAPE, "logit rules: too many rows x columns");
  hipLaunchKernelGGL((logit_rules_kernel<T, VEC, ITER>), dim3((unsigned)n), dim3(kRuleThreads), 0, st, a, chunks,
                     lowest);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

// Chunks of 1,024 columns where that makes up to 2,048 workgroups, 8 a CU, which then
// share out what one would do in turn; beyond, chunks of 4,096, so that a history is read
// once per 4,096 columns (chunks of 4,096 and of 1,024, us: 16 rows of 33,024 bf16 columns
// 6.5 and 4.6; 2 rows of 17,051 fp32 8.6 and 5.2; 64 rows of 33,024 7.1 and 7.0; but 120
// rows 10.2 and 11.3, 400 rows of 16,487 16.3 and 20.1).
template <class T>
static atspeed_status run_rules(const atspeed_logit_rules_args& a, bool vec, float lowest, hipStream_t st) {
  const bool small = a.n_cols <= 1024 || (long long)a.n_rows * ((a.n_cols + 1023) / 1024) <= 2048;
  if (vec) return small ? launch_rules<T, 4, 1>(a, lowest, st) : launch_rules<T, 4, 4>(a, lowest, st);
  return small ? launch_rules<T, 1, 4>(a, lowest, st) : launch_rules<T, 1, 16>(a, lowest, st);
}

// What the rules themselves need: the pointers that go together, and their counts.
atspeed_status check_rules(const atspeed_logit_rules_args& a) {
  if ((a.history != nullptr) != (a.hist_len != nullptr)) return fail(ATSPEED_E_INVALID, "history and hist_len go together");
  if (a.history && a.max_hist < 1) return fail(ATSPEED_E_INVALID, "max_hist must be >= 1");
  if (a.bias && a.n_bias < 1) return fail(ATSPEED_E_INVALID, "n_bias must be >= 1");
  if ((a.allowed != nullptr) != (a.state != nullptr)) return fail(ATSPEED_E_INVALID, "allowed and state go together");
  if (a.allowed && a.n_states < 1) return fail(ATSPEED_E_INVALID, "n_states must be >= 1");
  if (a.bias && a.bias_stride < a.n_cols) return fail(ATSPEED_E_SHAPE, "a row stride is below n_cols");
  return ATSPEED_OK;
}

atspeed_status logit_rules(const atspeed_logit_rules_args& a, float lowest, hipStream_t st) {
  if (a.dtype != ATSPEED_FP32 && a.dtype != ATSPEED_BF16) return fail(ATSPEED_E_INVALID, "dtype");
  if (a.B < 1 || a.B > kMaxRequests) return fail(ATSPEED_E_INVALID, "B must be 1..1024");
  if (a.n_rows < 0) return fail(ATSPEED_E_INVALID, "n_rows must be >= 0");
  if (a.n_cols < 1 || a.n_cols > (1 << 20)) return fail(ATSPEED_E_INVALID, "n_cols must be 1..2^20");
  if (a.n_rows == 0) return ATSPEED_OK;
  if (!a.logits || !a.out || !a.row_off) return fail(ATSPEED_E_INVALID, "logit rules: null pointer");
  ST_TRY(check_rules(a));
  if (a.node_token && a.max_nodes < 1) return fail(ATSPEED_E_INVALID, "max_nodes must be >= 1");
  if (a.node_token && a.mask && a.mask_words < 1) return fail(ATSPEED_E_INVALID, "mask_words must be >= 1");
  if (a.out_row && a.n_out_rows < 1) return fail(ATSPEED_E_INVALID, "n_out_rows must be >= 1");
  if (a.logits_stride < a.n_cols || a.out_stride < a.n_cols)
    return fail(ATSPEED_E_SHAPE, "a row stride is below n_cols");
  if ((const void*)a.out == a.logits &&
      (a.dtype != ATSPEED_FP32 || a.out_row || a.out_stride != a.logits_stride))
    return fail(ATSPEED_E_INVALID, "in place needs fp32 logits, one stride and no out_row");
  const int es = a.dtype == ATSPEED_BF16 ? 2 : 4;
  auto fits = [](const void* p, int64_t stride, int bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && stride % 4 == 0;
  };
  const bool vec = fits(a.logits, a.logits_stride, 4 * es) && fits(a.out, a.out_stride, 16) &&
                   (!a.bias || fits(a.bias, a.bias_stride, 16));
  return a.dtype == ATSPEED_BF16 ? run_rules<bf16_t>(a, vec, lowest, st) : run_rules<float>(a, vec, lowest, st);
}

}  // namespace atspeed

extern "C" atspeed_status atspeed_logit_rules(const atspeed_logit_rules_args* args, void* stream) {
  if (!args) return atspeed::fail(ATSPEED_E_INVALID, "args is null");
  return atspeed::logit_rules(*args, -INFINITY, (hipStream_t)stream);
}
