// Pages of forked requests (atspeed_page_fork), copies of pages (atspeed_page_copy) and
// accepted paths moved together (atspeed_kv_compact).
#include <algorithm>

#include "common.h"
#include "paged.h"

namespace atspeed {

typedef unsigned long long u64;

// ---------------------------------------------------------------- page tables
// What a page's holders are after the call depends on every row, so the work goes in steps
// that each end a launch:
//   clear   the pages' counters,
//   count   per page the old entries and the new full ones, and the lowest row that wants it
//           as its last page; the new tables are put down beside the old ones,
//   decide  how many pages of each piece of the pool come free; which rows copy, numbered,
//   write   tables, holders, free list.
// All sums are of whole numbers, so the atomics' order changes nothing.
constexpr int kForkThreads = 256;
constexpr int kForkRows = 8;         // consecutive rows of a thread that counts
constexpr int kNoRow = 0x7fffffff;

struct ForkArgs {
  atspeed_page_fork_args a;
  u64* holders;      // [n_pool] old entries << 32 | new full entries
  int* first;        // [n_pool] lowest row that wants the page as its last one
  int* next;         // [B, max_pages] the new tables, up to the last page
  int* gone;         // [pieces] pages of a piece of the pool that come free
  int* rank;         // [B] 1, 2, ... for the rows that copy, 0 for the others
  int* taker;        // [B] the rows that copy, in order
  int* total;        // [2] rows that copy; pages that were free
  int shift, piece, pieces;
};

struct ForkRow {
  int from, kept, before, full, over;   // source row (-1: none), tokens, old pages, full pages, tokens of the last one
  bool bad;
};
__device__ __forceinline__ int held_of(const ForkArgs& p, int j) {
  const int h = p.a.held[j];
  return h < 0 || h > (long long)p.a.max_pages << p.shift ? 0 : h;
}
__device__ __forceinline__ ForkRow row_of(const ForkArgs& p, int j) {
  ForkRow r;
  const int mine = held_of(p, j), tail = (1 << p.shift) - 1;
  r.from = p.a.src ? p.a.src[j] : j;
  r.bad = r.from < -1 || r.from >= p.a.B;
  const int there = r.bad || r.from < 0 ? 0 : held_of(p, r.from);
  r.kept = r.from == -1 ? 0 : p.a.keep ? p.a.keep[j] : there;
  r.bad = r.bad || r.kept < 0 || r.kept > there;
  if (r.bad) {
    r.from = j;
    r.kept = mine;
  }
  r.before = (int)(((long long)mine + tail) >> p.shift);
  r.full = r.kept >> p.shift;
  r.over = r.kept & tail;
  return r;
}

__global__ void __launch_bounds__(kForkThreads) fork_clear_kernel(ForkArgs p) {
  const int step = gridDim.x * kForkThreads;
  for (int i = blockIdx.x * kForkThreads + threadIdx.x; i < p.a.n_pool; i += step) {
    p.holders[i] = 0;
    p.first[i] = kNoRow;
  }
}

// A thread takes one column of a few consecutive rows: where these hold the same page, as
// the beams of one request do, it is counted once for all of them.
__global__ void __launch_bounds__(kForkThreads) fork_count_kernel(ForkArgs p, int columns) {
  const int c = blockIdx.x % columns * kForkThreads + threadIdx.x, j0 = blockIdx.x / columns * kForkRows;
  const int most = p.a.max_pages;
  int page = -1;
  u64 n = 0;
  auto add = [&](int q, u64 d) {
    if ((unsigned)q >= (unsigned)p.a.n_pool) return;
    if (q != page) {
      if (n) atomicAdd(&p.holders[page], n);
      page = q;
      n = 0;
    }
    n += d;
  };
  for (int j = j0; j < min(j0 + kForkRows, p.a.B); ++j) {
    const ForkRow r = row_of(p, j);
    if (c >= most) continue;
    if (c < r.before) add(p.a.block_table[(int64_t)j * most + c], 1ull << 32);
    if (r.from < 0 || c > r.full || (c == r.full && !r.over)) continue;
    const int q = p.a.block_table[(int64_t)r.from * most + c];
    p.next[(int64_t)j * most + c] = q;
    if (c < r.full) add(q, 1);
    else if ((unsigned)q < (unsigned)p.a.n_pool) atomicMin(&p.first[q], j);
  }
  if (n) atomicAdd(&p.holders[page], n);
}

// A page's further holders after the call (below 0: nobody holds it), and whether the first
// row that wants it as its last page takes it as it is.
__device__ __forceinline__ int left_of(const ForkArgs& p, int page, u64 h, bool& takes) {
  const int was = (int)(h >> 32), stays = (int)(unsigned)h;
  const int others = p.a.shared[page] - was;      // below 0: no holder but rows
  takes = stays == 0 && others < 0 && p.first[page] != kNoRow;
  return others + stays + takes;
}

__device__ __forceinline__ int sum_threads(int x, int* part) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < kForkThreads / 64; ++w) x += part[w];
  return x;
}
// Sum of the threads before this one, and of all.
__device__ __forceinline__ int scan_threads(int x, int* part, int* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = inc;
  __syncthreads();
  int before = inc - x, total = 0;
#pragma unroll
  for (int w = 0; w < kForkThreads / 64; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  *all = total;
  return before;
}

// Workgroup i < pieces: a piece of the pool; the last one: the rows.
__global__ void __launch_bounds__(kForkThreads) fork_decide_kernel(ForkArgs p) {
  __shared__ int part[kForkThreads / 64];
  if ((int)blockIdx.x < p.pieces) {
    const int begin = blockIdx.x * p.piece, end = min(begin + p.piece, p.a.n_pool);
    int n = 0;
    for (int i = begin + threadIdx.x; i < end; i += kForkThreads) {
      const u64 h = p.holders[i];
      bool takes;
      n += (h >> 32) && left_of(p, i, h, takes) < 0;
    }
    n = sum_threads(n, part);
    if (threadIdx.x == 0) p.gone[blockIdx.x] = n;
    return;
  }
  int before = 0;
  for (int j0 = 0; j0 < p.a.B; j0 += kForkThreads) {
    const int j = j0 + threadIdx.x;
    bool copies = false;
    if (j < p.a.B) {
      const ForkRow r = row_of(p, j);
      if (r.from >= 0 && r.over) {
        const int q = p.next[(int64_t)j * p.a.max_pages + r.full];
        if ((unsigned)q < (unsigned)p.a.n_pool) {
          bool takes;
          left_of(p, q, p.holders[q], takes);
          copies = !(takes && p.first[q] == j);
        }
      }
    }
    int all;
    const int at = before + scan_threads(copies, part, &all);
    if (j < p.a.B) p.rank[j] = copies ? at + 1 : 0;
    if (copies) p.taker[at] = j;
    before += all;
  }
  if (threadIdx.x == 0) {
    p.total[0] = before;
    p.total[1] = min(max(*p.a.n_free, 0), p.a.n_pool);
  }
}

// Workgroup i < pieces: holders and free list of a piece of the pool; the others: a row each.
// Of the stack of free pages -- those that were free, then the released ones in ascending
// order -- the k-th row that copies has the k-th from the top.
__global__ void __launch_bounds__(kForkThreads) fork_write_kernel(ForkArgs p) {
  __shared__ int part[kForkThreads / 64];
  const int tid = threadIdx.x, most = p.a.max_pages, piece = min((int)blockIdx.x, p.pieces);
  int ahead = 0, all = 0;
  for (int i = tid; i < p.pieces; i += kForkThreads) {
    const int n = p.gone[i];
    all += n;
    ahead += i < piece ? n : 0;
  }
  all = sum_threads(all, part);
  ahead = sum_threads(ahead, part);
  const int F = p.total[1], have = (int)min((long long)F + all, (long long)p.a.n_pool);
  const int top = have - min(p.total[0], have);
  if ((int)blockIdx.x < p.pieces) {
    const int begin = blockIdx.x * p.piece, end = min(begin + p.piece, p.a.n_pool);
    int s = F + ahead;
    for (int i0 = begin; i0 < end; i0 += kForkThreads) {
      const int i = i0 + tid;
      bool out = false;
      if (i < end) {
        const u64 h = p.holders[i];
        if (h >> 32) {
          bool takes;
          const int left = left_of(p, i, h, takes);
          out = left < 0;
          p.a.shared[i] = max(left, 0);
        }
      }
      int n;
      const int at = s + scan_threads(out, part, &n);
      if (out && at < top) p.a.free_pages[at] = i;
      if (out && at >= top && at < have) {
        const int j = p.taker[have - 1 - at];
        const ForkRow r = row_of(p, j);
        p.a.block_table[(int64_t)j * most + r.full] = i;
        p.a.copy_dst[j] = i;
      }
      s += n;
    }
    if (blockIdx.x == 0 && tid == 0) *p.a.n_free = top;
    return;
  }
  const int j = blockIdx.x - p.pieces, rank = p.rank[j];
  const ForkRow r = row_of(p, j);
  const bool copies = rank > 0 && rank <= have, refused = rank > have;
  for (int c = tid; c < r.full + (r.over && !rank); c += kForkThreads)
    if (r.from >= 0 && r.from != j) p.a.block_table[(int64_t)j * most + c] = p.next[(int64_t)j * most + c];
  if (tid == 0) {
    p.a.length[j] = refused ? r.full << p.shift : r.kept;
    p.a.refused[j] = r.bad ? 2 : refused;
    p.a.copy_src[j] = copies ? p.next[(int64_t)j * most + r.full] : -1;
    p.a.copy_len[j] = copies ? r.over : 0;
    if (!copies) {
      p.a.copy_dst[j] = -1;
    } else if (have - rank < F) {
      const int q = p.a.free_pages[have - rank];
      p.a.block_table[(int64_t)j * most + r.full] = q;
      p.a.copy_dst[j] = q;
    }
  }
}

// ---------------------------------------------------------------- moving tokens
struct MoveArgs {
  PagesDev kp, vp;
  int64_t k_layer, v_layer;    // bytes
  const int* src;              // page copies: pages and token counts
  const int* dst;
  const int* length;
  const int* table;            // paths: [B, max_pages], [B], [B, max_path], [B]
  const int* ctx;
  const int* path;
  const int* n_path;
  int layers, chunks, head_shift, page_shift, n_pool, max_pages, max_path;
};

constexpr int kMoveThreads = 256;

// A workgroup a copy and layer; 16-byte chunks of the page's first tokens, k and v.
__global__ void __launch_bounds__(kMoveThreads) page_copy_kernel(MoveArgs a) {
  const int i = blockIdx.x / a.layers, layer = blockIdx.x % a.layers;
  const int src = a.src[i], dst = a.dst[i];
  if ((unsigned)src >= (unsigned)a.n_pool || (unsigned)dst >= (unsigned)a.n_pool) return;
  const int n = min(a.length[i], 1 << a.page_shift) * a.chunks;
  const char* k = a.kp.data + layer * a.k_layer;
  const char* v = a.vp.data + layer * a.v_layer;
  for (int c = threadIdx.x; c < n; c += kMoveThreads) {
    const int token = c / a.chunks, in = c % a.chunks;
    const int64_t h = in >> a.head_shift, e = (in & ((1 << a.head_shift) - 1)) * 16;
    const int64_t ko = token * a.kp.token + h * a.kp.head + e, vo = token * a.vp.token + h * a.vp.head + e;
    const u32x4_t kk = *reinterpret_cast<const u32x4_t*>(k + src * a.kp.page + ko);
    const u32x4_t vv = *reinterpret_cast<const u32x4_t*>(v + src * a.vp.page + vo);
    *reinterpret_cast<u32x4_t*>(const_cast<char*>(k) + dst * a.kp.page + ko) = kk;
    *reinterpret_cast<u32x4_t*>(const_cast<char*>(v) + dst * a.vp.page + vo) = vv;
  }
}

// A workgroup a request and layer.  A thread moves its chunk of every token, in the path's
// order: a place is written only behind the moves that read it, since path[i] >= i.
constexpr int kMaxPath = 4096;

__global__ void __launch_bounds__(kMoveThreads) kv_compact_kernel(MoveArgs a) {
  __shared__ int from[kMaxPath], to[kMaxPath];     // cache slots
  const int b = blockIdx.x / a.layers, layer = blockIdx.x % a.layers;
  const int n = a.n_path[b], ctx = a.ctx[b], tail = (1 << a.page_shift) - 1;
  if (n < 1 || n > a.max_path || ctx < 0) return;
  const int* path = a.path + (int64_t)b * a.max_path;
  const int* table = a.table + (int64_t)b * a.max_pages;
  bool ok = true;
  auto slot_of = [&](long long at) {
    const long long page = at >> a.page_shift;
    const int q = page < a.max_pages ? table[page] : -1;
    if ((unsigned)q >= (unsigned)a.n_pool) ok = false;
    return (q << a.page_shift) + (int)(at & tail);
  };
  for (int i = threadIdx.x; i < n; i += kMoveThreads) {
    const int row = path[i];
    ok = ok && row > (i ? path[i - 1] : -1);
    if (!ok) break;
    from[i] = slot_of((long long)ctx + row);
    to[i] = slot_of((long long)ctx + i);
  }
  if (!__syncthreads_and(ok)) return;
  const char* k = a.kp.data + layer * a.k_layer;
  const char* v = a.vp.data + layer * a.v_layer;
  for (int c = threadIdx.x; c < 2 * a.chunks; c += kMoveThreads) {
    const bool of_v = c >= a.chunks;
    const PagesDev& p = of_v ? a.vp : a.kp;
    const int in = of_v ? c - a.chunks : c;
    const int64_t h = in >> a.head_shift, e = (in & ((1 << a.head_shift) - 1)) * 16;
    char* base = const_cast<char*>(of_v ? v : k) + h * p.head + e;
    auto at = [&](int slot) {
      return reinterpret_cast<u32x4_t*>(base + (int64_t)(slot >> a.page_shift) * p.page + (int64_t)(slot & tail) * p.token);
    };
    for (int i = 0; i < n; ++i)
      if (from[i] != to[i]) *at(to[i]) = *at(from[i]);
  }
}

static atspeed_status check_layers(int n_layers, int64_t k_layer, int64_t v_layer, int es) {
  if (n_layers < 1 || n_layers > 1024) return fail(ATSPEED_E_INVALID, "n_layers must be 1..1024");
  if ((k_layer * es) % 16 || (v_layer * es) % 16)
    return fail(ATSPEED_E_INVALID, "the layer strides must be multiples of 16 bytes");
  return ATSPEED_OK;
}

template <class A>
static atspeed_status move_args(const A& a, MoveArgs& p) {
  ST_TRY(check_head(a.dtype, a.d_head));
  ST_TRY(check_paging(a.page_size, a.n_pool));
  if (a.n_kv_heads < 1 || a.n_kv_heads > 1024) return fail(ATSPEED_E_INVALID, "n_kv_heads must be 1..1024");
  const int es = a.dtype == ATSPEED_BF16 ? 2 : 4;
  ST_TRY(check_pages(a.k_pages, es, "k_pages"));
  ST_TRY(check_pages(a.v_pages, es, "v_pages"));
  ST_TRY(check_layers(a.n_layers, a.k_layer_stride, a.v_layer_stride, es));
  p.kp = pages_dev(a.k_pages, es); p.vp = pages_dev(a.v_pages, es);
  p.k_layer = a.k_layer_stride * es; p.v_layer = a.v_layer_stride * es;
  const int cph = a.d_head * es / 16;
  p.layers = a.n_layers; p.chunks = a.n_kv_heads * cph; p.head_shift = log2_of(cph); p.page_shift = log2_of(a.page_size);
  p.n_pool = a.n_pool;
  return ATSPEED_OK;
}

static atspeed_status check_fork(const atspeed_page_fork_args& a) {
  if (a.B < 1 || a.B > kMaxRequests) return fail(ATSPEED_E_INVALID, "B must be 1..1024");
  ST_TRY(check_paging(a.page_size, a.n_pool));
  if (a.max_pages < 1) return fail(ATSPEED_E_INVALID, "max_pages must be >= 1");
  if ((long long)a.B * a.max_pages >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "B x max_pages must be below 2^31");
  if (!a.held || !a.block_table || !a.free_pages || !a.n_free || !a.shared || !a.length || !a.refused || !a.copy_src ||
      !a.copy_dst || !a.copy_len)
    return fail(ATSPEED_E_INVALID, "page fork: null pointer");
  const void* in[] = {a.held, a.keep, a.src};
  const void* out[] = {a.length, a.refused, a.copy_src, a.copy_dst, a.copy_len, a.n_free, a.shared, a.free_pages, a.block_table};
  for (const void* i : in)
    for (const void* o : out)
      if (i && i == o) return fail(ATSPEED_E_INVALID, "page fork: an output is one of the inputs");
  return ATSPEED_OK;
}

static size_t lay_out(ForkArgs& p, char* base) {
  const atspeed_page_fork_args& a = p.a;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = base ? base + at : nullptr;
    at += (bytes + 255) & ~(size_t)255;
    return q;
  };
  // at most 1,024 pieces, since every workgroup of the last step adds them up
  p.piece = std::max(1024, (a.n_pool + 1023) / 1024);
  p.pieces = (a.n_pool + p.piece - 1) / p.piece;
  p.shift = log2_of(a.page_size);
  p.holders = (u64*)take((size_t)a.n_pool * 8);
  p.first = (int*)take((size_t)a.n_pool * 4);
  p.next = (int*)take((size_t)a.B * a.max_pages * 4);
  p.gone = (int*)take((size_t)p.pieces * 4);
  p.rank = (int*)take((size_t)a.B * 4);
  p.taker = (int*)take((size_t)a.B * 4);
  p.total = (int*)take(8);
  return at;
}

}  // namespace atspeed

using namespace atspeed;

extern "C" {

atspeed_status atspeed_page_fork_workspace_bytes(const atspeed_page_fork_args* args, size_t* bytes) {
  if (!args || !bytes) return fail(ATSPEED_E_INVALID, "args or bytes is null");
  ST_TRY(check_fork(*args));
  ForkArgs p{};
  p.a = *args;
  *bytes = lay_out(p, nullptr);
  return ATSPEED_OK;
}

atspeed_status atspeed_page_fork(const atspeed_page_fork_args* args, void* workspace, size_t ws_bytes, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  ST_TRY(check_fork(*args));
  ForkArgs p{};
  p.a = *args;
  const int columns = (args->max_pages + kForkThreads - 1) / kForkThreads;
  const long long count = (long long)columns * ((args->B + kForkRows - 1) / kForkRows);
  if (count > kMaxGroups) return fail(ATSPEED_E_SHAPE, "page fork: too many rows x pages");
  const size_t need = lay_out(p, nullptr);
  if (!workspace || !aligned16(workspace) || ws_bytes < need)
    return fail(ATSPEED_E_WORKSPACE, "page fork: workspace is too small or not 16-byte aligned");
  lay_out(p, (char*)workspace);
  const hipStream_t st = (hipStream_t)stream;
  const int clear = std::min((args->n_pool + kForkThreads - 1) / kForkThreads, 1024);
  hipLaunchKernelGGL(fork_clear_kernel, dim3(clear), dim3(kForkThreads), 0, st, p);
  hipLaunchKernelGGL(fork_count_kernel, dim3((unsigned)count), dim3(kForkThreads), 0, st, p, columns);
  hipLaunchKernelGGL(fork_decide_kernel, dim3(p.pieces + 1), dim3(kForkThreads), 0, st, p);
  hipLaunchKernelGGL(fork_write_kernel, dim3(p.pieces + args->B), dim3(kForkThreads), 0, st, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

atspeed_status atspeed_page_copy(const atspeed_page_copy_args* args, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  MoveArgs p{};
  ST_TRY(move_args(*args, p));
  if (args->n < 0) return fail(ATSPEED_E_INVALID, "n must be >= 0");
  if (args->n == 0) return ATSPEED_OK;
  if (!args->src || !args->dst || !args->length) return fail(ATSPEED_E_INVALID, "page copy: null pointer");
  p.src = args->src; p.dst = args->dst; p.length = args->length;
  const long long groups = (long long)args->n * args->n_layers;
  if (groups > kMaxGroups) return fail(ATSPEED_E_SHAPE, "page copy: too many copies x layers");
  hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)groups), dim3(kMoveThreads), 0, (hipStream_t)stream, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

atspeed_status atspeed_kv_compact(const atspeed_kv_compact_args* args, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  MoveArgs p{};
  ST_TRY(move_args(*args, p));
  if (args->B < 1 || args->B > kMaxRequests) return fail(ATSPEED_E_INVALID, "B must be 1..1024");
  if (args->max_pages < 1) return fail(ATSPEED_E_INVALID, "max_pages must be >= 1");
  if (args->max_path < 1 || args->max_path > kMaxPath) return fail(ATSPEED_E_INVALID, "max_path must be 1..4096");
  if (!args->block_table || !args->ctx || !args->path || !args->n_path)
    return fail(ATSPEED_E_INVALID, "kv compact: null pointer");
  p.table = args->block_table; p.ctx = args->ctx; p.path = args->path; p.n_path = args->n_path;
  p.max_pages = args->max_pages; p.max_path = args->max_path;
  const long long groups = (long long)args->B * args->n_layers;
  hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)groups), dim3(kMoveThreads), 0, (hipStream_t)stream, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

}  // extern "C"
