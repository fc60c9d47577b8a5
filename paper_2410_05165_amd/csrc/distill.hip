// Distillation of a draft from a teacher's top logits: the loss (atspeed_distill_loss) and
// its gradient (atspeed_distill_grad).
//
// Both divergences live on n_tops + 1 buckets, the tops and the rest, and every column of
// the rest has the gradient d A q_v with one A a row.  So the loss needs one pass over the
// logits for their largest and the sums of their exponentials, the gradient one more that
// writes exp(z - largest) times a number of the row, and then the tops' own values.
//
// The rest's share of q is summed by itself, without the tops (a bit a column in LDS says
// which these are): as 1 - sum of the tops it would keep only what fp32 leaves of a small
// difference, and A = 1 - p_rest / q_rest with it.
#include <cfloat>
#include <cmath>

#include "common.h"
#include "paged.h"
#include "wave.h"

namespace atspeed {

constexpr int kMaxTops = 256;
constexpr float kNoTop = -0.f;   // in the place of a top's gradient, which is never -0: no top

template <class T>
__device__ __forceinline__ void unpack(const u32x4_t raw, float (&x)[16 / sizeof(T)]) {
  constexpr int VEC = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < VEC; ++i)
    x[i] = VEC == 4 ? __uint_as_float(raw[i]) : __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
}

// c: log2(e) / temperature.  exp2 of (z - top) * c with -infinity as 0 whatever top is.
__device__ __forceinline__ float weight_of(float z, float top, float c) {
  return z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((z - top) * c);
}

// Sum over the threads that have tops: those of a wave, or of four through LDS.
__device__ __forceinline__ double sum_tops(double x, bool one_wave, double* part) {
  x = wave_sum(x);
  if (one_wave) return x;
  __syncthreads();
  if ((threadIdx.x & 63) == 0 && threadIdx.x < kMaxTops) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// A workgroup a row.  Three barriers for up to 64 tops: the tops' bits and the teacher's
// largest logit, the teacher's sum, the row's largest and sum; then the tops' wave is alone.
// Bound by memory: 8,192 rows of 33,024 fp32 columns (1.08 GB) 232 us, 4.7 TB/s; 2,048 bf16 ones
// (135 MB) 32; 640 rows of 1,024 6.4, where it is the chain of loads, barriers and logarithms
// (with a barrier for every sum 271, 42 and 10.4).
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) distill_loss_kernel(atspeed_distill_loss_args a, float c) {
  constexpr int VEC = 16 / sizeof(T), WAVES = THREADS / 64, STEP = THREADS * VEC;
  extern __shared__ uint32_t bits[];               // a bit a column: a top
  __shared__ int index[kMaxTops], twice;
  __shared__ double far_of[kMaxTops], part[4], wave_top[WAVES], wave_all[WAVES];
  __shared__ float row_top[WAVES], row_sum[WAVES];
  const int r = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, m = a.n_tops, V = a.n_cols;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.logits_stride;
  float* saved = a.saved + (int64_t)r * (2 + m);

  // asked for at once: the row's first columns and the teacher's; thread j has top j
  auto load = [&](int v) {
    u32x4_t raw = {};
    if (v + VEC <= V) {
      raw = *reinterpret_cast<const u32x4_any_t*>(row + v);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        uint32_t x = sizeof(T) == 2 ? 0xff80u : 0xff800000u;       // -infinity
        if (v + i < V) x = VEC == 4 ? reinterpret_cast<const uint32_t*>(row)[v + i] : reinterpret_cast<const uint16_t*>(row)[v + i];
        raw[i * 4 / VEC] |= x << (VEC == 4 ? 0 : 16 * (i & 1));
      }
    }
    return raw;
  };
  u32x4_t ahead[2] = {load(tid * VEC), load(tid * VEC + STEP)};
  int mine = -1;
  float teacher = -INFINITY;
  if (tid < m) {
    mine = a.teacher_index[(int64_t)r * m + tid];
    teacher = St<T>::ld(static_cast<const T*>(a.teacher_logit) + (int64_t)r * m + tid);
  }
  const float weight = a.weight ? a.weight[r] : 1.f;
  const double tail = a.tail ? (double)a.tail[r] : -INFINITY, inv_t = 1.0 / (double)a.temperature;
  if (tid == 0) twice = 0;
  for (int i = tid; i < (V + 31) / 32; i += THREADS) bits[i] = 0;
  if ((unsigned)mine >= (unsigned)V || teacher == -INFINITY) mine = -1;
  const double t = mine >= 0 ? (double)teacher * inv_t : -INFINITY;
  const float z = mine >= 0 ? St<T>::ld(row + mine) : -INFINITY;
  double t_top = t;
  static_for<6>([&](auto s) { t_top = fmax(t_top, partner<s>(t_top)); });
  if ((tid & 63) == 0) wave_top[wave] = t_top;
  if (tid < m) index[tid] = mine;
  const bool counts = __syncthreads_or(mine >= 0) && weight != 0.f;
  if (!counts) {
    if (tid < 2) saved[tid] = 0.f;
    if (tid < m) saved[2 + tid] = kNoTop;
    if (tid == 0) a.loss[r] = 0.f;
    return;
  }
  if (mine >= 0 && (atomicOr(&bits[mine >> 5], 1u << (mine & 31)) >> (mine & 31) & 1)) twice = 1;
  t_top = tail;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) t_top = fmax(t_top, wave_top[w]);
  // NaN and +infinity among them go through to the loss, as those of the row's logits
  const double w = mine < 0 ? 0.0 : t < INFINITY ? exp_below(t, t_top) : NAN;
  const double w_rest = tail == -INFINITY ? 0.0 : tail < INFINITY ? exp_below(tail, t_top) : NAN;
  const double w_wave = wave_sum(w);
  if ((tid & 63) == 0) wave_all[wave] = w_wave;
  if (tid < m) far_of[tid] = t - t_top;
  __syncthreads();
  // one pass over the logits: the largest, and the sum of the others' exponentials
  float top = -INFINITY, sum = 0.f;
  for (int v0 = tid * VEC; __any(v0 < V); v0 += 2 * STEP) {
    u32x4_t raw[2] = {ahead[0], ahead[1]};
    if (v0 + 2 * STEP < V) ahead[0] = load(v0 + 2 * STEP);
    if (v0 + 3 * STEP < V) ahead[1] = load(v0 + 3 * STEP);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int v = v0 + h * STEP;
      if (v >= V) continue;
      float x[VEC];
      unpack<T>(raw[h], x);
      float most = x[0];
#pragma unroll
      for (int i = 1; i < VEC; ++i) most = max_nan(most, x[i]);
      if (!(most <= top)) {
        const float now = max_nan(most, top);
        if (top > -INFINITY) sum *= __builtin_amdgcn_exp2f((top - now) * c);
        top = now;
      }
      if (top == -INFINITY) continue;
      const uint32_t tops = (bits[v >> 5] >> (v & 31)) & ((1u << VEC) - 1);
      float some = 0.f;                            // vectors first: a thread's sum has few terms
      if (!__any(tops)) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) some += __builtin_amdgcn_exp2f((x[i] - top) * c);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) some += tops >> i & 1 ? 0.f : __builtin_amdgcn_exp2f((x[i] - top) * c);
      }
      sum += some;
    }
  }
  float z_top = wave_max_nan(top);
  const float w_sum = wave_sum(top > -INFINITY ? sum * __builtin_amdgcn_exp2f((top - z_top) * c) : 0.f);
  if ((tid & 63) == 0) {
    row_top[wave] = z_top;
    row_sum[wave] = w_sum;
  }
  __syncthreads();
  const bool one_wave = m <= 64;
  if (one_wave && wave) return;
  z_top = row_top[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) z_top = max_nan(z_top, row_top[i]);
  double w_all = w_rest;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) w_all += wave_all[i];
  const bool bad = !(z_top < INFINITY) || !(w_all == w_all);   // of the row's own or the teacher's
  if (bad) z_top = NAN;
  double rest = 0.0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i)
    if (row_top[i] > -INFINITY) rest += (double)(row_sum[i] * __builtin_amdgcn_exp2f((row_top[i] - z_top) * c));
  // p and its logarithm, which goes on where p is 0: (t - t_top) - log w_all.  Columns that were
  // named twice: the first one has the sum, its logarithm taken around their largest
  const double log_w = log(w_all);
  bool first = mine >= 0;
  double p = w, log_p = t - t_top;
  if (twice && mine >= 0) {
    for (int j = 0; j < m; ++j)
      if (index[j] == mine) {
        if (j < tid) first = false;
        log_p = fmax(log_p, far_of[j]);
      }
    double all_mine = 0.0;
    for (int j = 0; j < m; ++j)
      if (index[j] == mine) all_mine += exp_below(far_of[j], log_p);
    p = all_mine * exp_below(log_p, 0.0);
    log_p += log(all_mine);
  }
  p /= w_all;
  log_p -= log_w;
  const double e = mine >= 0 ? (double)weight_of(z, z_top, c) : 0.0;
  const double all = rest + sum_tops(first ? e : 0.0, one_wave, part);

  // the divergence, bucket by bucket
  const bool empty = all == 0.0;                   // no logit but -infinity: q is 0
  const double inv_all = 1.0 / all, q = empty ? 0.0 : e * inv_all, q_rest = empty ? 0.0 : rest * inv_all;
  const double p_rest = w_rest / w_all;
  const double log_all = log(all);
  const double log_q = z == -INFINITY ? -INFINITY : ((double)z - (double)z_top) * inv_t - log_all;
  const double log_qr = rest == 0.0 ? -INFINITY : log(rest) - log_all, log_pr = (tail - t_top) - log_w;
  double mass = 0.0, far = 0.0, mass_r = 0.0, far_r = 0.0;     // a bucket's weight, log of the quotient
  if (a.reverse) {
    mass = first && e > 0.0 ? q : 0.0;
    far = log_q - log_p;
    mass_r = rest > 0.0 ? q_rest : 0.0;
    far_r = log_qr - log_pr;
  } else {
    mass = first && p > 0.0 ? p : 0.0;
    far = log_p - log_q;
    mass_r = p_rest;
    far_r = log_pr - log_qr;
  }
  if (bad || !(all == all)) mass_r = far_r = NAN;
  const double loss = sum_tops(mass > 0.0 ? mass * far : 0.0, one_wave, part) + (mass_r == 0.0 ? 0.0 : mass_r * far_r);
  const double step = (double)weight * (double)a.temperature;
  double at_top = 0.0, a_rest = 0.0;
  if (a.reverse) {
    at_top = e > 0.0 ? q * (far - loss) : 0.0;
    a_rest = rest > 0.0 ? far_r - loss : 0.0;
  } else {
    at_top = q - p;
    a_rest = rest > 0.0 ? 1.0 - p_rest / q_rest : 0.0;
  }
  if (bad) at_top = a_rest = NAN;
  if (tid < m) saved[2 + tid] = mine >= 0 ? (float)(step * at_top) + 0.f : kNoTop;
  if (tid == 0) {
    // beyond fp32's range where the rest is next to nothing
    const double to_rest = all > 0.0 || bad ? step * a_rest / all : 0.0;
    saved[0] = z_top;
    saved[1] = fabs(to_rest) > FLT_MAX ? (float)copysign((double)FLT_MAX, to_rest) : (float)to_rest;
    a.loss[r] = (float)(step * (double)a.temperature * loss);
  }
}

// A workgroup a row and 4,096 columns.  Bound by memory: 8,192 rows of 33,024 fp32 columns
// (2.16 GB) 384 us, 2,048 bf16 ones (270 MB) 43.
constexpr int kDistThreads = 256;
constexpr int kGradVecs = 16;   // columns a thread

template <class T>
__global__ void __launch_bounds__(kDistThreads) distill_grad_kernel(atspeed_distill_grad_args a, float c, int chunks) {
  constexpr int VEC = 16 / sizeof(T), COLS = kDistThreads * kGradVecs;
  const int r = blockIdx.x / chunks, v0 = blockIdx.x % chunks * COLS, m = a.n_tops, V = a.n_cols, tid = threadIdx.x;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.logits_stride;
  T* out = static_cast<T*>(a.grad) + (int64_t)r * a.grad_stride;
  const float* saved = a.saved + (int64_t)r * (2 + m);
  const float g = a.grad_loss ? a.grad_loss[r] : 1.f;
  // a factor of the rest's size may have no fp32 product with a scaled loss's g: g then comes
  // behind the exponential, which may be 0
  const float top = saved[0], both = saved[1] == 0.f ? 0.f : saved[1] * g;
  const bool apart = !(fabsf(both) <= FLT_MAX);
  const float scale = apart ? saved[1] : both, behind = apart ? g : 1.f;
#pragma unroll
  for (int k = 0; k < kGradVecs / VEC; ++k) {
    const int v = v0 + (k * kDistThreads + tid) * VEC;
    if (v >= V) continue;
    if (v + VEC <= V) {
      float x[VEC];
      unpack<T>(*reinterpret_cast<const u32x4_any_t*>(row + v), x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = scale == 0.f ? 0.f : scale * weight_of(x[i], top, c) * behind;
      u32x4_t raw;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        raw[i] = VEC == 4 ? __float_as_uint(x[i])
                          : (uint32_t)f2bf(x[VEC == 4 ? 0 : 2 * i]) | (uint32_t)f2bf(x[VEC == 4 ? 0 : 2 * i + 1]) << 16;
      *reinterpret_cast<u32x4_any_t*>(out + v) = raw;
    } else {
      for (int i = v; i < V; ++i) St<T>::st(out + i, scale == 0.f ? 0.f : scale * weight_of(St<T>::ld(row + i), top, c) * behind);
    }
  }
  __syncthreads();               // the tops' own values come behind
  if (tid < m) {
    const int at = a.teacher_index[(int64_t)r * m + tid];
    const float x = saved[2 + tid];
    const bool is = __float_as_uint(x) != __float_as_uint(kNoTop);
    if (is && at >= v0 && at < min(v0 + COLS, V)) St<T>::st(out + at, x == 0.f ? 0.f : x * g);
  }
}

template <class T, int THREADS>
static atspeed_status launch_loss(const atspeed_distill_loss_args& a, size_t lds, float c, hipStream_t st) {
  if (lds > (48 << 10))
    HIP_TRY(hipFuncSetAttribute((const void*)distill_loss_kernel<T, THREADS>, hipFuncAttributeMaxDynamicSharedMemorySize, 1 << 17));
  hipLaunchKernelGGL((distill_loss_kernel<T, THREADS>), dim3(a.n_rows), dim3(THREADS), lds, st, a, c);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}
// Rows longer than 16,384 columns that leave CUs empty take workgroups of 1,024 (us, of 256
// and of 1,024: 16 rows of 131,072 bf16 columns 23.8 and 15.4, 64 of 33,024 10.5 and 9.0, 256 of
// them 11.1 and 9.9; but 512 of them 13.5 and 17.0, 256 of 8,192 6.6 and 7.7).
template <class T>
static atspeed_status run_loss(const atspeed_distill_loss_args& a, size_t lds, float c, hipStream_t st) {
  return a.n_cols > 16384 && a.n_rows <= 256 ? launch_loss<T, 1024>(a, lds, c, st) : launch_loss<T, 256>(a, lds, c, st);
}

static float exponent_scale(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

static atspeed_status check_distill(int dtype, int n_rows, int n_cols, int n_tops, float temperature) {
  if (dtype != ATSPEED_FP32 && dtype != ATSPEED_BF16) return fail(ATSPEED_E_INVALID, "dtype");
  if (n_rows < 0) return fail(ATSPEED_E_INVALID, "n_rows must be >= 0");
  if (n_cols < 1 || n_cols > (1 << 20)) return fail(ATSPEED_E_INVALID, "n_cols must be 1..2^20");
  if (n_tops < 1 || n_tops > kMaxTops) return fail(ATSPEED_E_INVALID, "n_tops must be 1..256");
  if (!(temperature > 0.f) || !(temperature < INFINITY) || !(exponent_scale(temperature) < INFINITY))
    return fail(ATSPEED_E_INVALID, "temperature must be positive, its reciprocal finite");
  return ATSPEED_OK;
}

}  // namespace atspeed

using namespace atspeed;

extern "C" {

atspeed_status atspeed_distill_loss(const atspeed_distill_loss_args* args, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  const atspeed_distill_loss_args& a = *args;
  ST_TRY(check_distill(a.dtype, a.n_rows, a.n_cols, a.n_tops, a.temperature));
  if (a.reverse && !a.tail) return fail(ATSPEED_E_INVALID, "the reverse form needs the teacher's tail");
  if (a.n_rows == 0) return ATSPEED_OK;
  if (!a.logits || !a.teacher_logit || !a.teacher_index || !a.loss || !a.saved)
    return fail(ATSPEED_E_INVALID, "distill loss: null pointer");
  if (a.logits_stride < a.n_cols && a.n_rows > 1) return fail(ATSPEED_E_SHAPE, "a row stride is below n_cols");
  if (a.n_rows > kMaxGroups) return fail(ATSPEED_E_SHAPE, "distill loss: too many rows");
  const size_t lds = (size_t)(a.n_cols + 31) / 32 * 4;
  const float c = exponent_scale(a.temperature);
  return a.dtype == ATSPEED_BF16 ? run_loss<bf16_t>(a, lds, c, (hipStream_t)stream) : run_loss<float>(a, lds, c, (hipStream_t)stream);
}

atspeed_status atspeed_distill_grad(const atspeed_distill_grad_args* args, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  const atspeed_distill_grad_args& a = *args;
  ST_TRY(check_distill(a.dtype, a.n_rows, a.n_cols, a.n_tops, a.temperature));
  if (a.n_rows == 0) return ATSPEED_OK;
  if (!a.logits || !a.teacher_index || !a.saved || !a.grad) return fail(ATSPEED_E_INVALID, "distill grad: null pointer");
  if ((a.logits_stride < a.n_cols || a.grad_stride < a.n_cols) && a.n_rows > 1)
    return fail(ATSPEED_E_SHAPE, "a row stride is below n_cols");
  if (a.grad == a.logits) return fail(ATSPEED_E_INVALID, "distill grad: an output is one of the inputs");
  const int cols = kDistThreads * kGradVecs, chunks = (a.n_cols + cols - 1) / cols;
  const long long groups = (long long)a.n_rows * chunks;
  if (groups > kMaxGroups) return fail(ATSPEED_E_SHAPE, "distill grad: too many rows x columns");
  const float c = exponent_scale(a.temperature);
  const dim3 grid((unsigned)groups), threads(kDistThreads);
  if (a.dtype == ATSPEED_BF16)
    hipLaunchKernelGGL((distill_grad_kernel<bf16_t>), grid, threads, 0, (hipStream_t)stream, a, c, chunks);
  else
    hipLaunchKernelGGL((distill_grad_kernel<float>), grid, threads, 0, (hipStream_t)stream, a, c, chunks);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

}  // extern "C"
