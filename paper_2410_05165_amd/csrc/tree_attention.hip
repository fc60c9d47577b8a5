// Tree attention over a paged cache (atspeed_tree_attention).
#include <algorithm>
#include <cmath>

#include "common.h"
#include "paged.h"

namespace atspeed {

struct TreeAttnArgs {
  const char* q;
  int64_t q_row, q_head;       // bytes
  PagesDev k, v;
  const int* table;
  const int* row_off;
  const int* ctx;
  const uint64_t* mask;
  char* out;
  int64_t o_row, o_head;       // bytes
  float* lse;
  int B, n_rows, H, G, max_pages, n_pool, max_new, words, shift;
  float scale;
};

// One wave per row and head: 64 keys at a time, a key per lane for the scores and
// dims lane, lane + 64 of the output for the sums; one pass with a running maximum.
template <class T, int DH>
__global__ void __launch_bounds__(64) tree_attn_simple_kernel(TreeAttnArgs a) {
  __shared__ float qs[DH];
  const int r = blockIdx.x / a.H, h = blockIdx.x % a.H, lane = threadIdx.x;
  if (r >= a.row_off[a.B]) return;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.row_off[mid] <= r) lo = mid; else hi = mid;
  }
  const int b = lo, i = r - a.row_off[b], kvh = h / a.G;
  if (i >= a.max_new) return;
  const int count = a.row_off[b + 1] - a.row_off[b];
  const long long ctx = a.ctx[b];
  const long long cap = (long long)a.max_pages << a.shift;
  const long long total = ctx < 0 ? 0 : min(ctx + (a.mask ? min(count, a.words * 64) : i + 1), cap);
  const T* q = reinterpret_cast<const T*>(a.q + r * a.q_row + h * a.q_head);
  for (int d = lane; d < DH; d += 64) qs[d] = St<T>::ld(q + d);
  __syncthreads();
  float m = -INFINITY, sum = 0.f, o[(DH + 63) / 64] = {};
  for (long long k0 = 0; k0 < total; k0 += 64) {
    const long long key = k0 + lane;
    bool see = key < total;
    int page = -1;
    if (see && key >= ctx && a.mask) {
      const int j = (int)(key - ctx);
      see = (a.mask[(int64_t)r * a.words + (j >> 6)] >> (j & 63)) & 1;
    }
    if (see) {
      page = a.table[(int64_t)b * a.max_pages + (key >> a.shift)];
      see = (unsigned)page < (unsigned)a.n_pool;
    }
    float s = -INFINITY;
    const int64_t tok = key & ((1 << a.shift) - 1);
    if (see) {
      const T* kp = reinterpret_cast<const T*>(a.k.data + page * a.k.page + tok * a.k.token + kvh * a.k.head);
      float dot = 0.f;
      for (int d = 0; d < DH; ++d) dot += qs[d] * St<T>::ld(kp + d);
      s = dot * a.scale;
    }
    float mx = s;
    for (int w = 1; w < 64; w <<= 1) mx = fmaxf(mx, __shfl_xor(mx, w));
    const float mnew = fmaxf(m, mx), ref = mnew == -INFINITY ? 0.f : mnew;
    const float alpha = m == -INFINITY ? 0.f : expf(m - ref);
    const float p = see ? expf(s - ref) : 0.f;
    float ps = p;
    for (int w = 1; w < 64; w <<= 1) ps += __shfl_xor(ps, w);
    sum = sum * alpha + ps;
    m = mnew;
    for (int n = 0; n < (DH + 63) / 64; ++n) o[n] *= alpha;
    for (int e = 0; e < 64; ++e) {
      if (!__shfl((int)see, e)) continue;
      const float pe = __shfl(p, e);
      const int pg = __shfl(page, e);
      const int64_t te = (k0 + e) & ((1 << a.shift) - 1);
      const T* vp = reinterpret_cast<const T*>(a.v.data + pg * a.v.page + te * a.v.token + kvh * a.v.head);
      for (int n = 0; n < (DH + 63) / 64; ++n)
        if (n * 64 + lane < DH) o[n] += pe * St<T>::ld(vp + n * 64 + lane);
    }
  }
  const bool none = sum == 0.f;
  T* out = reinterpret_cast<T*>(a.out + r * a.o_row + h * a.o_head);
  for (int n = 0; n < (DH + 63) / 64; ++n)
    if (n * 64 + lane < DH) St<T>::st(out + n * 64 + lane, none ? 0.f : o[n] / sum);
  if (a.lse && lane == 0) a.lse[(int64_t)r * a.H + h] = none ? -INFINITY : m + logf(sum);
}

static atspeed_status check_attention(const atspeed_tree_attention_args* args) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  const atspeed_tree_attention_args& a = *args;
  ST_TRY(check_head(a.dtype, a.d_head));
  ST_TRY(check_paging(a.page_size, a.n_pool));
  if (a.B < 1 || a.B > kMaxRequests) return fail(ATSPEED_E_INVALID, "B must be 1..1024");
  if (a.n_rows < 0 || a.max_ctx < 0 || a.max_new < 0) return fail(ATSPEED_E_INVALID, "n_rows, max_ctx and max_new must be >= 0");
  if (a.n_heads < 1 || a.n_heads > 1024 || a.n_kv_heads < 1 || a.n_heads % a.n_kv_heads)
    return fail(ATSPEED_E_SHAPE, "n_heads must be 1..1024 and a multiple of n_kv_heads");
  if (a.max_pages < 1) return fail(ATSPEED_E_INVALID, "max_pages must be >= 1");
  if (!std::isfinite(a.scale)) return fail(ATSPEED_E_INVALID, "scale must be finite");
  if (a.mask && a.mask_words < 1) return fail(ATSPEED_E_INVALID, "mask_words must be >= 1");
  if ((long long)a.n_rows * a.n_heads >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "n_rows x n_heads must be below 2^31");
  return ATSPEED_OK;
}

}  // namespace atspeed

using namespace atspeed;

extern "C" {

atspeed_status atspeed_tree_attention_workspace_bytes(const atspeed_tree_attention_args* args, size_t* bytes) {
  if (!bytes) return fail(ATSPEED_E_INVALID, "bytes is null");
  ST_TRY(check_attention(args));
  *bytes = 0;
  return ATSPEED_OK;
}

atspeed_status atspeed_tree_attention(const atspeed_tree_attention_args* args, void* workspace, size_t ws_bytes,
                                      void* stream) {
  ST_TRY(check_attention(args));
  const atspeed_tree_attention_args& a = *args;
  if (a.n_rows == 0 || a.max_new == 0) return ATSPEED_OK;
  const int es = a.dtype == ATSPEED_BF16 ? 2 : 4;
  ST_TRY(check_rows(a.q, a.q_row_stride, a.q_head_stride, es, "q"));
  ST_TRY(check_rows(a.out, a.out_row_stride, a.out_head_stride, es, "out"));
  ST_TRY(check_pages(a.k_pages, es, "k_pages"));
  ST_TRY(check_pages(a.v_pages, es, "v_pages"));
  if (!a.block_table || !a.row_off || !a.ctx) return fail(ATSPEED_E_INVALID, "tree attention: null pointer");
  TreeAttnArgs p{};
  p.q = (const char*)a.q; p.q_row = a.q_row_stride * es; p.q_head = a.q_head_stride * es;
  p.k = pages_dev(a.k_pages, es); p.v = pages_dev(a.v_pages, es);
  p.table = a.block_table; p.row_off = a.row_off; p.ctx = a.ctx; p.mask = a.mask;
  p.out = (char*)a.out; p.o_row = a.out_row_stride * es; p.o_head = a.out_head_stride * es;
  p.lse = a.lse;
  p.B = a.B; p.n_rows = a.n_rows; p.H = a.n_heads; p.G = a.n_heads / a.n_kv_heads;
  p.max_pages = a.max_pages; p.n_pool = a.n_pool; p.max_new = a.max_new; p.words = a.mask_words;
  p.shift = log2_of(a.page_size); p.scale = a.scale;
  const dim3 grid((unsigned)(a.n_rows * (long long)a.n_heads)), block(64);
  hipStream_t st = (hipStream_t)stream;
  if (es == 2) {
    if (a.d_head == 64) hipLaunchKernelGGL((tree_attn_simple_kernel<bf16_t, 64>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((tree_attn_simple_kernel<bf16_t, 128>), grid, block, 0, st, p);
  } else {
    if (a.d_head == 32) hipLaunchKernelGGL((tree_attn_simple_kernel<float, 32>), grid, block, 0, st, p);
    else if (a.d_head == 64) hipLaunchKernelGGL((tree_attn_simple_kernel<float, 64>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((tree_attn_simple_kernel<float, 128>), grid, block, 0, st, p);
  }
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

}  // extern "C"
