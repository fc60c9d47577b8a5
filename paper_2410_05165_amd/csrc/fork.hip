// Pages of forked requests (atspeed_page_fork), copies of pages (atspeed_page_copy) and
// accepted paths moved together (atspeed_kv_compact).
#include <algorithm>
#include <climits>

#include "common.h"
#include "paged.h"

namespace atspeed {

typedef unsigned long long u64;

// ---------------------------------------------------------------- page tables
// What becomes of a page depends on every row, so the work has steps, each behind the one
// before:
//   count   shared[page] loses one for each old entry and gains one for each new full one; the
//           new tables are put down beside the old ones, which other rows still read,
//   claim   a last page that is left without a holder (-1; below it where rows held the page
//           more often than shared said) goes to the lowest row that wants it,
//   decide  the other rows that want one copy; they are numbered, and so are the pages that
//           come free (below 0) in pieces of the pool,
//   write   tables, holders, free list.
// Sums and minima of whole numbers: the order of the atomics changes nothing.  Launches of
// their own for count, claim and decide (one workgroup), and write; one workgroup does it all
// where there is little to do.  Bound by latency, chains of dependent loads: the ten beams of one
// user 6.4 us, 1,000 rows of up to 257 pages 7.7 + 9.0 + 5.7 (counters of their own, cleared first,
// and a scan of the pool by its pieces took four launches, 17 and 33 us).  The scan in `decide`
// grows with the pool, 8,192 pages a step, and not with what was touched: the call takes 21 us with
// 20,000 pages, 28 with 60,000, 41 with 140,000, 245 with a million.
constexpr int kForkThreads = 256, kForkOne = 1024;
// What one workgroup takes by itself: rows, and entries of the tables and pages (us, one launch
// and three: 10 rows of 6 entries 6.3 and 13.4, 100 of 40 13.1 and 15.8; but 320 of 13 20.7 and
// 15.8, 400 of 20 26.2 and 15.9).
constexpr int kForkRows = 128, kForkFew = 4096;
constexpr int kPieces = 1024;        // of the pool, at most
constexpr int kRun = 8;              // consecutive rows of a thread that counts

struct ForkArgs {
  atspeed_page_fork_args a;
  int* next;         // [B, max_pages] the new tables, up to the last page
  int* last;         // [B] the page that a row wants as its last one, -1: none
  int* gone;         // [pieces + 1] pages that come free before a piece of the pool, and in all
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
  r.kept = p.a.keep ? p.a.keep[j] : -1;
  r.bad = r.from < -1 || r.from >= p.a.B;
  const int there = r.bad || r.from < 0 ? 0 : held_of(p, r.from);
  r.kept = r.from == -1 ? 0 : p.a.keep ? r.kept : there;
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
// Waits until what the workgroup stored, added and loaded is done.
__device__ __forceinline__ void sync_memory() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}
// What this launch may have changed.
__device__ __forceinline__ int fresh(const int* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool is_page(const ForkArgs& p, int q) { return (unsigned)q < (unsigned)p.a.n_pool; }

// Column c of rows j0 .. j1 - 1 (row: theirs, from j0 on).  Where these hold the same page, as
// the beams of one request do, it is counted once for all of them.
template <int RUN>
__device__ __forceinline__ void count_column(const ForkArgs& p, const ForkRow* row, int c, int j0, int j1) {
  const int most = p.a.max_pages;
  int was[RUN], will[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    was[i] = will[i] = -1;
    if (j0 + i >= j1) continue;
    const ForkRow& r = row[i];
    if (c < r.before) was[i] = p.a.block_table[(int64_t)(j0 + i) * most + c];
    if (r.from >= 0 && c < r.full + (r.over > 0)) {
      const int q = p.a.block_table[(int64_t)r.from * most + c];
      p.next[(int64_t)(j0 + i) * most + c] = q;
      if (c < r.full) will[i] = q;
      else p.last[j0 + i] = is_page(p, q) ? q : -1;
    }
    if (c == 0 && (r.from < 0 || !r.over)) p.last[j0 + i] = -1;
  }
  int page = -1, n = 0;
  auto add = [&](int q, int d) {
    if (!is_page(p, q)) return;
    if (q != page) {
      if (n) atomicAdd(&p.a.shared[page], n);
      page = q;
      n = 0;
    }
    n += d;
  };
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    add(was[i], -1);
    add(will[i], 1);
  }
  if (n) atomicAdd(&p.a.shared[page], n);
}

// Sum of the threads before this one, and of all.
template <int THREADS>
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
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  *all = total;
  return before;
}

// claim and decide, by one workgroup of kForkOne threads: a thread a row, a wave 64 pages at a
// time.  Rows that want the same page meet in a table of pages in LDS, half full at most.
constexpr int kSlots = 2 * kForkOne;

__device__ __forceinline__ void decide(const ForkArgs& p) {
  __shared__ int part[kForkOne / 64], gone[kPieces], page[kSlots], lowest[kSlots];
  const int j = threadIdx.x, B = p.a.B, lane = j & 63, chunks = (int)(((long long)p.a.n_pool + 63) / 64);
  const int q = j < B ? fresh(&p.last[j]) : -1;
  for (int i = j; i < kSlots; i += kForkOne) {
    page[i] = -1;
    lowest[i] = kForkOne;
  }
  gone[j] = 0;
  const bool may = q >= 0 && fresh(&p.a.shared[q]) < 0;
  __syncthreads();
  int slot = (unsigned)(q * 0x9E3779B1u) >> 21;
  if (may) {
    for (;; slot = (slot + 1) & (kSlots - 1)) {
      const int there = atomicCAS(&page[slot], -1, q);
      if (there == -1 || there == q) break;
    }
    atomicMin(&lowest[slot], j);
  }
  for (int c0 = j >> 6; c0 < chunks; c0 += 8 * (kForkOne / 64)) {
    int left[8];
#pragma unroll
    for (int o = 0; o < 8; ++o) {
      const unsigned i = (unsigned)(c0 + o * (kForkOne / 64)) * 64 + lane;     // past 2^31 behind the largest pools
      left[o] = i < (unsigned)p.a.n_pool ? fresh(&p.a.shared[i]) : 0;
    }
#pragma unroll
    for (int o = 0; o < 8; ++o) {
      const int n = __popcll(__ballot(left[o] < 0));
      if (n && lane == 0) atomicAdd(&gone[(unsigned)(c0 + o * (kForkOne / 64)) * 64 / p.piece], n);
    }
  }
  sync_memory();                           // nobody looks at the pool any more
  const bool takes = may && lowest[slot] == j, copies = q >= 0 && !takes;
  if (takes) {
    p.a.shared[q] = 0;
    atomicSub(&gone[q / p.piece], 1);
  }
  int all;
  const int at = scan_threads<kForkOne>(copies, part, &all);
  if (j < B) p.rank[j] = copies ? at + 1 : 0;
  if (copies) p.taker[at] = j;
  if (j == 0) {
    p.total[0] = all;
    p.total[1] = min(max(*p.a.n_free, 0), p.a.n_pool);
  }
  const int ahead = scan_threads<kForkOne>(gone[j], part, &all);
  if (j < p.pieces) p.gone[j] = ahead;
  if (j == 0) p.gone[p.pieces] = all;
}

// Of the stack of free pages -- those that were free, then the released ones in ascending
// order -- the k-th row that copies has the k-th from the top.
struct Stack {
  int F, have, top;
};
__device__ __forceinline__ Stack stack_of(const ForkArgs& p) {
  Stack s;
  s.F = fresh(&p.total[1]);
  s.have = (int)min((long long)s.F + fresh(&p.gone[p.pieces]), (long long)p.a.n_pool);
  s.top = s.have - min(fresh(&p.total[0]), s.have);
  return s;
}
// Holders and free list of a piece of the pool, a wave.
template <class Row>
__device__ __forceinline__ void write_piece(const ForkArgs& p, const Stack& s, int i, int lane, Row row) {
  const unsigned begin = (unsigned)i * p.piece, end = min(begin + p.piece, (unsigned)p.a.n_pool);
  long long at = (long long)s.F + fresh(&p.gone[i]);
  for (unsigned c0 = begin; c0 < end; c0 += 64) {
    const unsigned c = c0 + lane;
    const int left = c < end ? fresh(&p.a.shared[c]) : 0;
    const u64 out = __ballot(left < 0);
    if (left < 0) {
      p.a.shared[c] = 0;
      const long long place = at + __popcll(out & ((1ull << lane) - 1));
      if (place < s.top) {
        p.a.free_pages[place] = (int)c;
      } else if (place < s.have) {
        const int j = fresh(&p.taker[s.have - 1 - place]);
        p.a.block_table[(int64_t)j * p.a.max_pages + row(j).full] = (int)c;
        p.a.copy_dst[j] = (int)c;
      }
    }
    at += __popcll(out);
  }
}
// A row's table and outputs, a wave.
__device__ __forceinline__ void write_row(const ForkArgs& p, const Stack& s, int j, int lane, const ForkRow& r) {
  const int rank = fresh(&p.rank[j]), most = p.a.max_pages;
  const bool copies = rank > 0 && rank <= s.have, refused = rank > s.have;
  if (r.from >= 0 && r.from != j) {
    const int n = r.full + (r.over && !rank);
    for (int c = lane; c < n; c += 64) p.a.block_table[(int64_t)j * most + c] = p.next[(int64_t)j * most + c];
  }
  if (lane) return;
  p.a.length[j] = refused ? r.full << p.shift : r.kept;
  p.a.refused[j] = r.bad ? 2 : refused;
  p.a.copy_src[j] = copies ? p.next[(int64_t)j * most + r.full] : -1;
  p.a.copy_len[j] = copies ? r.over : 0;
  if (!copies) {
    p.a.copy_dst[j] = -1;
  } else if (s.have - rank < s.F) {
    const int q = p.a.free_pages[s.have - rank];
    p.a.block_table[(int64_t)j * most + r.full] = q;
    p.a.copy_dst[j] = q;
  }
}

__global__ void __launch_bounds__(kForkThreads) fork_count_kernel(ForkArgs p, int columns) {
  __shared__ ForkRow row[kRun];
  const int c = blockIdx.x % columns * kForkThreads + threadIdx.x, j0 = blockIdx.x / columns * kRun;
  if (threadIdx.x < kRun && j0 + (int)threadIdx.x < p.a.B) row[threadIdx.x] = row_of(p, j0 + threadIdx.x);
  __syncthreads();
  if (c < p.a.max_pages) count_column<kRun>(p, row, c, j0, min(j0 + kRun, p.a.B));
}

__global__ void __launch_bounds__(kForkOne) fork_decide_kernel(ForkArgs p) {
  decide(p);
}

// A wave a piece of the pool, then a wave a row.
__global__ void __launch_bounds__(kForkThreads) fork_write_kernel(ForkArgs p) {
  const int i = __builtin_amdgcn_readfirstlane(blockIdx.x * (kForkThreads / 64) + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const Stack s = stack_of(p);
  if (i < p.pieces) write_piece(p, s, i, lane, [&](int j) { return row_of(p, j); });
  else if (i < p.pieces + p.a.B) write_row(p, s, i - p.pieces, lane, row_of(p, i - p.pieces));
  if (i == 0 && lane == 0) *p.a.n_free = s.top;
}

__global__ void __launch_bounds__(kForkOne) fork_one_kernel(ForkArgs p) {
  __shared__ ForkRow row[kForkOne];
  const int B = p.a.B, most = p.a.max_pages, lane = threadIdx.x & 63;
  if ((int)threadIdx.x < B) row[threadIdx.x] = row_of(p, threadIdx.x);
  __syncthreads();
  for (int i = threadIdx.x; i < B * most; i += kForkOne) count_column<1>(p, row + i / most, i % most, i / most, B);
  sync_memory();
  decide(p);
  sync_memory();
  const Stack s = stack_of(p);
  for (int i = threadIdx.x >> 6; i < p.pieces; i += kForkOne / 64)
    write_piece(p, s, i, lane, [&](int j) -> const ForkRow& { return row[j]; });
  for (int j = threadIdx.x >> 6; j < B; j += kForkOne / 64) write_row(p, s, j, lane, row[j]);
  if (threadIdx.x == 0) *p.a.n_free = s.top;
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
  const int* held;             // [B], null: not known
  int* keep;                   // [B], null: nobody asks
  int layers, chunks, head_shift, page_shift, n_pool, max_pages, max_path;
};

constexpr int kMoveThreads = 256;

// A workgroup a copy and layer; 16-byte chunks of the page's first tokens, k and v.  Bound by
// memory: 320 last pages of 16 tokens in 32 layers of 8 heads of 128 (603 MB moved) 101 us, above
// the 4.9 TB/s of a 2 GiB copy, since part of it stays in the last cache.
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

// A workgroup a request and layer.  A thread moves its chunk of every token, eight tokens at a
// time in the path's order: a place is written only behind the moves that read it, since
// path[i] >= i.  Bound by memory and the chain length, path, table, tokens: up to eight of 300
// nodes of 128 users in 32 layers of 8 heads of 128 (111 MB) 27.8 us (token by token 31).
constexpr int kMaxPath = 4096;

__global__ void __launch_bounds__(kMoveThreads) kv_compact_kernel(MoveArgs a) {
  __shared__ int from[kMaxPath], to[kMaxPath];     // cache slots
  const int b = blockIdx.x / a.layers, layer = blockIdx.x % a.layers;
  const int n = a.n_path[b], ctx = a.ctx[b], tail = (1 << a.page_shift) - 1;
  const int held = a.held ? a.held[b] : INT_MAX;
  const bool says = a.keep && layer == 0 && threadIdx.x == 0;
  if (says) a.keep[b] = ctx < 0 ? held : ctx;
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
    ok = ok && row > (i ? path[i - 1] : -1) && (long long)ctx + row < held;
    if (!ok) break;
    from[i] = slot_of((long long)ctx + row);
    to[i] = slot_of((long long)ctx + i);
  }
  if (!__syncthreads_and(ok)) return;
  if (says) a.keep[b] = ctx + n;
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
    for (int i0 = 0; i0 < n; i0 += 8) {
      u32x4_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *at(from[min(i0 + i, n - 1)]);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + i < n && from[i0 + i] != to[i0 + i]) *at(to[i0 + i]) = x[i];
    }
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
  p.piece = 256;
  while (p.piece < ((long long)a.n_pool + kPieces - 1) / kPieces) p.piece *= 2;
  p.pieces = (int)(((long long)a.n_pool + p.piece - 1) / p.piece);
  p.shift = log2_of(a.page_size);
  p.next = (int*)take((size_t)a.B * a.max_pages * 4);
  p.last = (int*)take((size_t)a.B * 4);
  p.gone = (int*)take((size_t)(p.pieces + 1) * 4);
  p.rank = (int*)take((size_t)a.B * 4);
  p.taker = (int*)take((size_t)a.B * 4);
  p.total = (int*)take(8);
  return at;
}

static atspeed_status compact(const atspeed_kv_compact_args* args, const int32_t* length, int32_t* keep, void* stream) {
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
  p.held = length; p.keep = keep;
  const long long groups = (long long)args->B * args->n_layers;
  hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)groups), dim3(kMoveThreads), 0, (hipStream_t)stream, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
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
  const int columns = (int)(((long long)args->max_pages + kForkThreads - 1) / kForkThreads);
  const long long count = (long long)columns * ((args->B + kRun - 1) / kRun);
  if (count > kMaxGroups) return fail(ATSPEED_E_SHAPE, "page fork: too many rows x pages");
  const size_t need = lay_out(p, nullptr);
  if (!workspace || !aligned16(workspace) || ws_bytes < need)
    return fail(ATSPEED_E_WORKSPACE, "page fork: workspace is too small or not 16-byte aligned");
  lay_out(p, (char*)workspace);
  const hipStream_t st = (hipStream_t)stream;
  if (args->B <= kForkRows && args->B * (long long)args->max_pages <= kForkFew && args->n_pool <= kForkFew) {
    hipLaunchKernelGGL(fork_one_kernel, dim3(1), dim3(kForkOne), 0, st, p);
  } else {
    hipLaunchKernelGGL(fork_count_kernel, dim3((unsigned)count), dim3(kForkThreads), 0, st, p, columns);
    hipLaunchKernelGGL(fork_decide_kernel, dim3(1), dim3(kForkOne), 0, st, p);
    const int waves = kForkThreads / 64;
    hipLaunchKernelGGL(fork_write_kernel, dim3((p.pieces + args->B + waves - 1) / waves), dim3(kForkThreads), 0, st, p);
  }
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
  return compact(args, nullptr, nullptr, stream);
}

atspeed_status atspeed_kv_compact_keep(const atspeed_kv_compact_args* args, const int32_t* length, int32_t* keep, void* stream) {
  if (!length || !keep) return fail(ATSPEED_E_INVALID, "kv compact: length or keep is null");
  if (args)
    for (const void* in : {(const void*)args->block_table, (const void*)args->ctx, (const void*)args->path,
                           (const void*)args->n_path, (const void*)length})
      if (in == keep) return fail(ATSPEED_E_INVALID, "kv compact: an output is one of the inputs");
  return compact(args, length, keep, stream);
}

}  // extern "C"
