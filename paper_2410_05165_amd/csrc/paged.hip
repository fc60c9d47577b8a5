// Step plan of a paged cache (atspeed_page_plan) and the append of new rows to it
// (atspeed_kv_append).
#include <algorithm>

#include "common.h"
#include "paged.h"

namespace atspeed {

// ---------------------------------------------------------------- step plan
// A few running sums over the requests (rows, released pages, wanted pages, granted
// pages) and then independent entries: table entries, free-list entries and rows,
// each of which finds its request by a binary search in those sums.  Every
// workgroup takes the sums for itself (up to 1,024 requests, 12 KB read from L2), so
// one launch does it all; nothing it reads is written by another workgroup:
//   - held, keep, add, n_free and parents are inputs that no output overlaps;
//   - pages are read from table entries of requests that do not take any (or before
//     the ones they take) and written to entries that are taken;
//   - of the free stack S (free_pages, then the released pages) the takers read
//     entries from the new top on, and the entries written lie below it.
// Bound by latency: three dependent loads (lengths, table or free list, parents).  5.0 us
// for one user's 30 nodes, 11.4 for 1,024 users with trees of up to 110 (9.6 for chains).
constexpr int kPlanThreads = 256;
constexpr int kPlanItems = kMaxRequests / kPlanThreads;

struct PlanArgs {
  atspeed_page_plan_args a;
  int shift, words;
};

// Exclusive running sum over the workgroup's items (kPlanItems consecutive ones a
// thread), in place; returns the total.
template <class T>
__device__ __forceinline__ T block_scan(T (&x)[kPlanItems], T* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T sum = 0;
#pragma unroll
  for (int i = 0; i < kPlanItems; ++i) sum += x[i];
  T inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = inc;
  __syncthreads();
  T before = inc - sum, total = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
#pragma unroll
  for (int i = 0; i < kPlanItems; ++i) {
    const T y = x[i];
    x[i] = before;
    before += y;
  }
  return total;
}

// Last b in [0, B) with off[b] <= i (off ascending from 0, i below its end).
__device__ __forceinline__ int owner(const int* off, int B, int i) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(PlanArgs p) {
  const atspeed_page_plan_args& a = p.a;
  __shared__ int row_off[kMaxRequests + 1], gone_off[kMaxRequests + 1], take_off[kMaxRequests + 1];
  __shared__ int before_s[kMaxRequests], after_s[kMaxRequests], keep_s[kMaxRequests];   // keep: -1 where refused
  __shared__ long long part64[kPlanThreads / 64];
  __shared__ int part32[kPlanThreads / 64];
  const int tid = threadIdx.x, B = a.B, most = a.max_pages, shift = p.shift;
  const int tail = (1 << shift) - 1;
  const bool first = blockIdx.x == 0;

  int held[kPlanItems], keep[kPlanItems], add[kPlanItems], refused[kPlanItems];
  long long rows[kPlanItems];
#pragma unroll
  for (int i = 0; i < kPlanItems; ++i) {
    const int b = tid * kPlanItems + i;
    const bool in = b < B;
    held[i] = in ? a.held[b] : 0;
    keep[i] = in ? a.keep[b] : 0;
    add[i] = in ? a.add[b] : 0;
    rows[i] = max(add[i], 0);
  }
  const int F = min(max(*a.n_free, 0), a.n_pool);
  const long long all_rows = block_scan(rows, part64);
  int gone[kPlanItems], want[kPlanItems], need[kPlanItems], before[kPlanItems], after[kPlanItems];
#pragma unroll
  for (int i = 0; i < kPlanItems; ++i) {
    const long long top = (long long)keep[i] + add[i];
    const long long was = ((long long)held[i] + tail) >> shift, will = (top + tail) >> shift;
    const bool bad = held[i] < 0 || keep[i] < 0 || keep[i] > held[i] || add[i] < 0 || was > most || will > most ||
                     top > 0x7fffffffLL ||
                     (a.parent && add[i] > a.max_nodes) || rows[i] + add[i] > a.max_rows;
    before[i] = bad ? 0 : (int)was;
    after[i] = bad ? 0 : (int)will;
    refused[i] = bad ? 2 : 0;
    gone[i] = max(before[i] - after[i], 0);
    want[i] = need[i] = max(after[i] - before[i], 0);
  }
  const int R = block_scan(gone, part32);
  block_scan(want, part32);
  const int have = (int)min((long long)F + R, (long long)a.n_pool);
  int take[kPlanItems];
#pragma unroll
  for (int i = 0; i < kPlanItems; ++i) {
    if (need[i] > 0 && (long long)want[i] + need[i] > have) refused[i] = 1;
    take[i] = refused[i] ? 0 : need[i];
  }
  const int T = block_scan(take, part32);
  if (tid == 0) {
    row_off[B] = (int)min(all_rows, (long long)a.max_rows);
    gone_off[B] = R;
    take_off[B] = T;
  }
#pragma unroll
  for (int i = 0; i < kPlanItems; ++i) {
    const int b = tid * kPlanItems + i;
    if (b >= B) continue;
    row_off[b] = (int)min(rows[i], (long long)a.max_rows);
    gone_off[b] = gone[i];
    take_off[b] = take[i];
    before_s[b] = before[i];
    after_s[b] = after[i];
    keep_s[b] = refused[i] ? -1 : keep[i];
    if (first) {
      a.refused[b] = refused[i];
      a.length[b] = refused[i] ? held[i] : keep[i] + add[i];
      a.ctx[b] = refused[i] ? -1 : keep[i];
      a.row_off[b] = (int)min(rows[i], (long long)a.max_rows);
    }
  }
  __syncthreads();
  const int n_rows = row_off[B], top = have - T;   // top: the new n_free
  if (first && tid == 0) {
    a.row_off[B] = n_rows;
    *a.n_free_out = top;
  }
  // entry j of the released pages, and entry s of the stack
  auto released = [&](int j) {
    const int b = owner(gone_off, B, j);
    return a.block_table[(size_t)b * most + after_s[b] + (j - gone_off[b])];
  };
  auto stack = [&](int s) { return s < F ? a.free_pages[s] : released(s - F); };

  const int step = gridDim.x * kPlanThreads, at = blockIdx.x * kPlanThreads + tid;
  for (int t = at; t < T; t += step) {
    const int b = owner(take_off, B, t);
    a.block_table[(size_t)b * most + before_s[b] + (t - take_off[b])] = stack(have - 1 - t);
  }
  for (int s = F + at; s < top; s += step) a.free_pages[s] = released(s - F);

  for (int r = at; r < a.max_rows; r += step) {
    int user = -1, pos = -1, slot = -1, ts = -1, b = 0, i = 0, depth = 0;
    if (r < n_rows) {
      b = owner(row_off, B, r);
      user = b;
      i = r - row_off[b];
      // a request of more rows than nodes (refused) has no place for the others: they would be the next one's
      ts = !a.parent ? i : i < a.max_nodes ? b * a.max_nodes + i : -1;
      if (keep_s[b] >= 0) {
        const int at_pos = keep_s[b] + i, pg = at_pos >> shift;
        // pages the request had are in its table, the others where the table entries come from
        const int page = pg < before_s[b] ? a.block_table[(size_t)b * most + pg]
                                          : stack(have - 1 - (take_off[b] + pg - before_s[b]));
        if ((unsigned)page < (unsigned)a.n_pool) slot = (page << shift) + (at_pos & tail);
        pos = at_pos;
        if (a.parent) {
          // the path must go down in index to a root
          const int* par = a.parent + (size_t)b * a.max_nodes;
          int cur = i;
          for (depth = 1;; ++depth) {
            const int up = par[cur];
            if (up == -1) break;
            if (up < 0 || up >= cur) {
              depth = 0;
              break;
            }
            cur = up;
          }
          pos = depth ? keep_s[b] + depth - 1 : -1;
        }
      }
    }
    a.row_user[r] = user;
    a.row_pos[r] = pos;
    a.slot[r] = slot;
    a.tree_slot[r] = ts;
    if (a.parent) {
      // indices fall along the path, so one word at a time is complete
      uint64_t* m = a.mask + (size_t)r * p.words;
      const int* par = a.parent + (size_t)b * a.max_nodes;
      int cur = depth ? i : -1;
      for (int w = p.words - 1; w >= 0; --w) {
        uint64_t bits = 0;
        while (cur >= w * 64) {
          bits |= 1ull << (cur & 63);
          cur = par[cur];
        }
        m[w] = bits;
      }
    }
  }
}

// ---------------------------------------------------------------- append
// One 16-byte chunk of k and one of v per thread and step; consecutive threads take
// consecutive chunks of a row, rows of few chunks share a workgroup.  Bound by memory:
// chunks of up to 1,024 rows x 32 users, 8 heads of 128 (99 MB), 16.0 us, above the
// 4.95 TB/s of a 2 GiB copy, since part of it stays in the last cache; 60 rows x 32 users,
// 32 heads (27 MB), 5.2.
struct AppendArgs {
  const char* k;
  const char* v;
  int64_t k_row, k_head, v_row, v_head;   // bytes
  PagesDev kp, vp;
  const int* slot;
  int n_rows, chunks, head_shift, page_shift, row_threads;
  unsigned n_slots;
};

__global__ void __launch_bounds__(256) kv_append_kernel(AppendArgs a) {
  const int per = 256 / a.row_threads;                   // rows of a workgroup
  const int r = blockIdx.x * per + threadIdx.x / a.row_threads;
  if (r >= a.n_rows) return;
  const int slot = a.slot[r];
  if ((unsigned)slot >= a.n_slots) return;
  const int64_t page = slot >> a.page_shift, token = slot & ((1 << a.page_shift) - 1);
  char* kd = const_cast<char*>(a.kp.data) + page * a.kp.page + token * a.kp.token;
  char* vd = const_cast<char*>(a.vp.data) + page * a.vp.page + token * a.vp.token;
  const char* ks = a.k + (int64_t)r * a.k_row;
  const char* vs = a.v + (int64_t)r * a.v_row;
  for (int c = threadIdx.x & (a.row_threads - 1); c < a.chunks; c += a.row_threads) {
    const int64_t h = c >> a.head_shift, e = (c & ((1 << a.head_shift) - 1)) * 16;
    const u32x4_t kk = *reinterpret_cast<const u32x4_t*>(ks + h * a.k_head + e);
    const u32x4_t vv = *reinterpret_cast<const u32x4_t*>(vs + h * a.v_head + e);
    *reinterpret_cast<u32x4_t*>(kd + h * a.kp.head + e) = kk;
    *reinterpret_cast<u32x4_t*>(vd + h * a.vp.head + e) = vv;
  }
}

}  // namespace atspeed

using namespace atspeed;

extern "C" {

atspeed_status atspeed_page_plan(const atspeed_page_plan_args* args, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  const atspeed_page_plan_args& a = *args;
  if (a.B < 1 || a.B > kMaxRequests) return fail(ATSPEED_E_INVALID, "B must be 1..1024");
  ST_TRY(check_paging(a.page_size, a.n_pool));
  if (a.max_pages < 1 || a.max_rows < 0) return fail(ATSPEED_E_INVALID, "max_pages must be >= 1 and max_rows >= 0");
  if ((long long)a.B * a.max_pages >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "B x max_pages must be below 2^31");
  if (!a.held || !a.keep || !a.add || !a.block_table || !a.free_pages || !a.n_free || !a.n_free_out || !a.length ||
      !a.ctx || !a.refused || !a.row_off)
    return fail(ATSPEED_E_INVALID, "page plan: null pointer");
  if (a.max_rows > 0 && (!a.row_user || !a.row_pos || !a.slot || !a.tree_slot))
    return fail(ATSPEED_E_INVALID, "page plan: null row output");
  if (a.parent) {
    if (a.max_nodes < 1 || a.max_nodes > 4096) return fail(ATSPEED_E_INVALID, "max_nodes must be 1..4096");
    if (!a.mask && a.max_rows > 0) return fail(ATSPEED_E_INVALID, "page plan: parents without a mask output");
  }
  const void* in[] = {a.held, a.keep, a.add, a.n_free};
  const void* out[] = {a.length, a.ctx, a.refused, a.n_free_out, a.row_off, a.row_user, a.row_pos, a.slot, a.tree_slot};
  for (const void* i : in)
    for (const void* o : out)
      if (i == o) return fail(ATSPEED_E_INVALID, "page plan: an output is one of the inputs");
  PlanArgs p{a, log2_of(a.page_size), (a.max_nodes + 63) / 64};
  const long long work = std::max<long long>({a.max_rows, a.B, 1});
  const int grid = (int)std::min<long long>((work + kPlanThreads - 1) / kPlanThreads, 1024);
  hipLaunchKernelGGL(page_plan_kernel, dim3(grid), dim3(kPlanThreads), 0, (hipStream_t)stream, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

atspeed_status atspeed_kv_append(const atspeed_kv_append_args* args, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  const atspeed_kv_append_args& a = *args;
  ST_TRY(check_head(a.dtype, a.d_head));
  ST_TRY(check_paging(a.page_size, a.n_pool));
  if (a.n_rows < 0 || a.n_kv_heads < 1 || a.n_kv_heads > 1024)
    return fail(ATSPEED_E_INVALID, "n_rows must be >= 0 and n_kv_heads 1..1024");
  if (a.n_rows == 0) return ATSPEED_OK;
  const int es = a.dtype == ATSPEED_BF16 ? 2 : 4;
  ST_TRY(check_rows(a.k, a.k_row_stride, a.k_head_stride, es, "k"));
  ST_TRY(check_rows(a.v, a.v_row_stride, a.v_head_stride, es, "v"));
  ST_TRY(check_pages(a.k_pages, es, "k_pages"));
  ST_TRY(check_pages(a.v_pages, es, "v_pages"));
  if (!a.slot) return fail(ATSPEED_E_INVALID, "slot is null");
  AppendArgs p{};
  p.k = (const char*)a.k; p.v = (const char*)a.v;
  p.k_row = a.k_row_stride * es; p.k_head = a.k_head_stride * es;
  p.v_row = a.v_row_stride * es; p.v_head = a.v_head_stride * es;
  p.kp = pages_dev(a.k_pages, es); p.vp = pages_dev(a.v_pages, es);
  p.slot = a.slot; p.n_rows = a.n_rows;
  const int cph = a.d_head * es / 16;
  p.chunks = a.n_kv_heads * cph; p.head_shift = log2_of(cph); p.page_shift = log2_of(a.page_size);
  p.row_threads = 1;
  while (p.row_threads < p.chunks && p.row_threads < 256) p.row_threads *= 2;
  p.n_slots = (unsigned)a.page_size * (unsigned)a.n_pool;
  const int per = 256 / p.row_threads;
  const long long groups = (a.n_rows + (long long)per - 1) / per;
  if (groups > kMaxGroups) return fail(ATSPEED_E_SHAPE, "append: too many rows x heads");
  hipLaunchKernelGGL(kv_append_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

}  // extern "C"
