// The k best continuations of each request's beams over the vocabulary
// (atspeed_beam_select).
//
// Within a row the order is that of the logits, so a first kernel reads every logit once
// and leaves the normaliser's sum and the k best logits of each part of a row; a second one
// ranks a request's lists by score[r] - log sum + logit.
//
// Scores of different beams are compared, so the normaliser must not move them past each
// other: it is taken in 64 bits (exponentials to 1.1e-12), where fp32 exponentials (1e-7 of the sum)
// would swap one pair of neighbours in some thousand lists.  64-bit vector instructions
// run at the rate of 32-bit ones here.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "paged.h"

namespace atspeed {

typedef unsigned long long u64;
typedef u32x4_t u32x4_any_t __attribute__((aligned(2)));   // 16 bytes at any element

constexpr int kBeamThreads = 256, kBeamWaves = kBeamThreads / 64;
constexpr int kLane = 16;              // columns of a lane in a tile
constexpr int kTile = 64 * kLane;      // columns of a wave's tile
constexpr int kMaxBeams = 256;         // k

// e^d for d from -740 to 0, to 1.1e-12 of itself and 1 at 0: 2^n by the exponent, 2^r for r on
// [-1/2, 1/2] by the polynomial of degree 8 that is 1 at 0 and has the least largest relative
// error (found by exchanging its extrema).  The difference of two fp32 logits is exact enough however large they are.
constexpr float kLeast = -740.f;
__device__ __forceinline__ double exp_64(double d) {
  constexpr double log2e = 0x1.71547652b82fep0;
  const double shifted = __builtin_fma(d, log2e, 0x1.8p52);   // its low bits are the nearest whole number
  const double r = __builtin_fma(d, log2e, 0x1.8p52 - shifted);
  double p = 0x1.663487d8abc81p-20;
  p = __builtin_fma(p, r, 0x1.00ee071c7c030p-16);
  p = __builtin_fma(p, r, 0x1.4306c1165a375p-13);
  p = __builtin_fma(p, r, 0x1.5d872975c4ed2p-10);
  p = __builtin_fma(p, r, 0x1.3b2ab7f3b3217p-7);
  p = __builtin_fma(p, r, 0x1.c6b08defc25fdp-5);
  p = __builtin_fma(p, r, 0x1.ebfbdff7c5a79p-3);
  p = __builtin_fma(p, r, 0x1.62e42fef7a78bp-1);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_ldexp(p, (int)(unsigned)__double_as_longlong(shifted));
}
// e^(x - top), x <= top
__device__ __forceinline__ double exp_below(double x, double top) { return exp_64(fmax(x - top, (double)kLeast)); }

// fp32 (no NaN) to whole numbers of the same order, -0 as 0; and back.
__device__ __forceinline__ uint32_t order_of(float x) { return float_order_key(x + 0.f); }
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
// A column's place among its row's: by the logit, then the lower column.
__device__ __forceinline__ u64 column_key(uint32_t order, int col) { return ((u64)order << 32) | (0xffffffffu - (unsigned)col); }
__device__ __forceinline__ int column_of(u64 key) { return (int)(0xffffffffu - (unsigned)key); }
__device__ __forceinline__ u64 order64(double x) {
  const u64 u = (u64)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// Largest of two, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_max_nan(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = max_nan(x, __shfl_xor(x, o));
  return x;
}

// A lane's 16 columns of a tile: 16-byte loads of consecutive lanes, wherever the row begins.
template <class T>
__device__ __forceinline__ int column_at(int lane, int e) {
  constexpr int VEC = 16 / sizeof(T);
  return (e / VEC) * (64 * VEC) + lane * VEC + e % VEC;
}
template <class T>
__device__ __forceinline__ void load_tile(const T* row, int c0, int n_cols, int lane, float (&x)[kLane]) {
  constexpr int VEC = 16 / sizeof(T);
  if (c0 + kTile <= n_cols) {
#pragma unroll
    for (int v = 0; v < kLane / VEC; ++v) {
      const u32x4_t raw = *reinterpret_cast<const u32x4_any_t*>(row + c0 + (v * 64 + lane) * VEC);
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        x[v * VEC + i] = VEC == 4 ? __uint_as_float(raw[i])
                                  : __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < kLane; ++e) {
      const int c = c0 + column_at<T>(lane, e);
      x[e] = c < n_cols ? St<T>::ld(row + c) : -INFINITY;
    }
  }
}

// Largest t such that at least k of the wave's N numbers a lane are >= t, in steps of
// 2^low (0 if there are fewer than k numbers above 0).
template <int N, class U>
__device__ __forceinline__ U kth_largest(const U (&x)[N], int k, int low) {
  U t = 0;
#pragma unroll 1
  for (int bit = 8 * sizeof(U) - 1; bit >= low; --bit) {
    const U at = t | ((U)1 << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popcll(__ballot(x[i] >= at));
    if (n >= k) t = at;
  }
  return t;
}

// A wave's best columns so far, up to P * 64 of them in LDS, in no order.
template <int P>
struct Pool {
  static constexpr int CAP = P * 64;
  u64* key;
  int n;
  u64 least;   // columns at or below it are not among the wave's k best

  // Keeps the k best.
  __device__ __forceinline__ void cut(int k, int lane) {
    u64 x[P];
    uint32_t hi[P];
    wave_sync();
#pragma unroll
    for (int i = 0; i < P; ++i) {
      x[i] = i * 64 + lane < n ? key[i * 64 + lane] : 0;
      hi[i] = (uint32_t)(x[i] >> 32);
    }
    const uint32_t t = kth_largest<P>(hi, k, 0);
    int above = 0, level = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      above += __popcll(__ballot(hi[i] > t));
      level += __popcll(__ballot(hi[i] == t));
    }
    u64 from = (u64)t << 32;
    if (above + level > k) {                    // equal logits: the lowest columns
      uint32_t lo[P];
#pragma unroll
      for (int i = 0; i < P; ++i) lo[i] = hi[i] == t ? (uint32_t)x[i] : 0;
      from |= kth_largest<P>(lo, k - above, 0);
    }
    wave_sync();
    n = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const u64 in = __ballot(x[i] >= from && x[i]);
      if (x[i] >= from && x[i]) key[n + __popcll(in & ((1ull << lane) - 1))] = x[i];
      n += __popcll(in);
    }
    least = from - 1;
  }

  // Takes in a tile's columns; k and 64 more have room.
  template <class T>
  __device__ __forceinline__ void add(const float (&x)[kLane], int c0, int k, int lane) {
    uint32_t todo = 0;
#pragma unroll
    for (int e = 0; e < kLane; ++e)
      if (x[e] > -INFINITY && order_of(x[e]) >= (uint32_t)(least >> 32)) todo |= 1u << e;
    while (__any(todo)) {
      bool full = false;
#pragma unroll
      for (int e = 0; e < kLane; ++e) {
        const u64 mine = column_key(order_of(x[e]), c0 + column_at<T>(lane, e));
        const bool is = (todo >> e & 1) && mine > least;
        const u64 in = __ballot(is);
        full = full || n + __popcll(in) > CAP;
        if (full || !in) continue;
        if (is) key[n + __popcll(in & ((1ull << lane) - 1))] = mine;
        n += __popcll(in);
        todo &= ~(1u << e);
      }
      if (!full) break;
      cut(k, lane);
    }
  }
};

struct BeamArgs {
  atspeed_beam_select_args a;
  u64* list;        // [n_rows, parts, k] the best columns, best first
  double2* stat;    // [n_rows, parts] largest logit and sum of exponentials; NaN: the row has no candidates
  int* len;         // [n_rows, parts]
  int parts, tiles; // parts of a row, tiles of a part
};

// Sorts key[0 .. n) with the payloads after it, n a power of two, largest key first, equal
// ones by the lower payload, by the whole workgroup.
template <bool PAY>
__device__ __forceinline__ void sort_desc(u64* key, u64* pay, int n) {
  for (int size = 2; size <= n; size <<= 1)
    for (int step = size >> 1; step; step >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < n / 2; i += kBeamThreads) {
        const int a = 2 * i - (i & (step - 1)), b = a + step;
        const u64 x = key[a], y = key[b];
        const bool ahead = x > y || (PAY && x == y && pay[a] < pay[b]);
        if (ahead == ((a & size) != 0) && (x != y || PAY)) {
          key[a] = y;
          key[b] = x;
          if (PAY) {
            const u64 p = pay[a];
            pay[a] = pay[b];
            pay[b] = p;
          }
        }
      }
    }
  __syncthreads();
}

template <class T, int P, bool PROBS>
__global__ void __launch_bounds__(kBeamThreads) beam_rows_kernel(BeamArgs p) {
  extern __shared__ u64 smem[];
  __shared__ float s_top[kBeamWaves];
  __shared__ double s_sum[kBeamWaves];
  __shared__ int s_n[kBeamWaves];
  const atspeed_beam_select_args& a = p.a;
  const int r = blockIdx.x / p.parts, part = blockIdx.x % p.parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (r >= a.row_off[a.B] || (a.done && a.done[r])) return;
  const int k = a.k, n_cols = a.n_cols;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.logits_stride;
  Pool<P> pool{smem + wave * Pool<P>::CAP, 0, 0};
  float top = -INFINITY;
  double sum = 0.0;
  bool bad = false;

  const int end = min((part + 1) * p.tiles, (n_cols + kTile - 1) / kTile);
  for (int tile = part * p.tiles + wave; tile < end; tile += kBeamWaves) {
    const int c0 = tile * kTile;
    float x[kLane], most[4];
    load_tile(row, c0, n_cols, lane, x);
#pragma unroll
    for (int g = 0; g < 4; ++g)
      most[g] = max_nan(max_nan(x[4 * g], x[4 * g + 1]), max_nan(x[4 * g + 2], x[4 * g + 3]));
    const float mine = max_nan(max_nan(most[0], most[1]), max_nan(most[2], most[3]));
    if (PROBS) {
      bad |= !(mine < INFINITY);
    } else {
      if (__any(!(mine <= top))) {
        const float now = wave_max_nan(max_nan(mine, top));
        if (top > -INFINITY) sum *= exp_below(top, now);
        top = now;
      }
      if (top > -INFINITY) {
        const float least = top + kLeast;             // below it nothing is left of the exponential
#pragma unroll
        for (int e = 0; e < kLane; ++e) sum += exp_64((double)fmaxf(x[e], least) - (double)top);
      }
    }
    // the first tile: fewer than k of its columns lie above this bound, of 256 groups' largest
    if (tile == part * p.tiles + wave) {
      uint32_t o[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) o[g] = most[g] > -INFINITY ? order_of(most[g]) : 0;
      const uint32_t t = kth_largest<4>(o, k, 16);
      pool.least = t ? ((u64)t << 32) - 1 : 0;
    }
    if (__any(mine > -INFINITY && order_of(mine) >= (uint32_t)(pool.least >> 32))) pool.template add<T>(x, c0, k, lane);
  }
  if (pool.n > k) pool.cut(k, lane);
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (PROBS) {
    top = 0.f;
    sum = __any(bad) ? NAN : 1.0;
  }
  if (lane == 0) {
    s_top[wave] = top;
    s_sum[wave] = sum;
    s_n[wave] = pool.n;
  }
  __syncthreads();

  // the part's statistics, and its k best in order
  if (threadIdx.x == 0) {
    float all = s_top[0];
    for (int w = 1; w < kBeamWaves; ++w) all = max_nan(all, s_top[w]);
    double total = 0.0;
    for (int w = 0; w < kBeamWaves; ++w)
      if (s_top[w] > -INFINITY || PROBS) total += s_sum[w] * exp_below(s_top[w], all);
    p.stat[blockIdx.x] = {(double)all, all < INFINITY ? total : NAN};
  }
  u64* sorted = smem + kBeamWaves * Pool<P>::CAP;
  int n = 0, size = 64;
#pragma unroll
  for (int w = 0; w < kBeamWaves; ++w) {
    if (w == wave)
      for (int i = lane; i < s_n[w]; i += 64) sorted[n + i] = pool.key[i];
    n += s_n[w];
  }
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += kBeamThreads) sorted[i] = 0;
  sort_desc<false>(sorted, nullptr, size);
  n = min(n, k);
  for (int i = threadIdx.x; i < n; i += kBeamThreads) p.list[(int64_t)blockIdx.x * k + i] = sorted[i];
  if (threadIdx.x == 0) p.len[blockIdx.x] = n;
}

// ---------------------------------------------------------------- ranking a request's lists
// A workgroup a request.  Rounds: every list whose next entry may still count gives a few,
// all that came are sorted, the k best stay, and the k-th is the bound of the next round.
// Entries are taken best first, so a list is left at its first one below the bound.
constexpr int kJoinPool = 2048, kJoinLists = 1024;

__global__ void __launch_bounds__(kBeamThreads) beam_join_kernel(BeamArgs p) {
  __shared__ u64 key[kJoinPool], pay[kJoinPool];   // the score's order; row << 32 | column + 1
  __shared__ double base[kJoinLists];              // of a row: score - log sum
  __shared__ short at[kJoinLists], len[kJoinLists];
  __shared__ int s_n, s_more;
  const atspeed_beam_select_args& a = p.a;
  const int b = blockIdx.x, tid = threadIdx.x, k = a.k, parts = p.parts;
  const int r1 = min(min(a.row_off[b + 1], a.row_off[a.B]), a.n_rows);   // rows that the first kernel read
  int r0 = max(a.row_off[b], 0);
  const int group = max(1, kJoinLists / parts);
  int n = 0;
  for (; r0 < r1; r0 += group) {
    const int rows = min(group, r1 - r0), lists = rows * parts;
    __syncthreads();
    for (int i = tid; i < rows; i += kBeamThreads) {
      const int r = r0 + i;
      const double score = a.score ? (double)a.score[r] : 0.0;
      double x = score;
      bool none = !(fabs(score) < INFINITY);
      if (!(a.done && a.done[r])) {
        const double2* st = p.stat + (int64_t)r * parts;
        double all = -INFINITY, total = 0.0;
        for (int q = 0; q < parts; ++q)
          if (st[q].x > all) all = st[q].x;
        for (int q = 0; q < parts; ++q) {
          // a part whose largest logit is -infinity has sum 0; NaN stays
          if (st[q].x > -INFINITY) total += st[q].y * exp_below(st[q].x, all);
          else if (!(st[q].x == -INFINITY)) total = NAN;
        }
        if (a.log_probs) {
          if (!(total == total)) none = true;
        } else {
          x = score - (all + log(total));
          if (!(fabs(x) < INFINITY)) none = true;
        }
      }
      base[i] = none ? NAN : x;
    }
    __syncthreads();
    for (int l = tid; l < lists; l += kBeamThreads) {
      const int i = l / parts, r = r0 + i;
      const bool ended = a.done && a.done[r];
      at[l] = 0;
      len[l] = !(base[i] == base[i]) ? 0 : ended ? l % parts == 0 : p.len[(int64_t)r * parts + l % parts];
    }
    for (;;) {
      __syncthreads();
      if (tid == 0) {
        s_n = n;
        s_more = 0;
      }
      __syncthreads();
      const u64 low_key = n == k ? key[k - 1] : 0, low_pay = n == k ? pay[k - 1] : 0;
      const int quota = max(1, min((2 * k + lists - 1) / lists, (kJoinPool - k) / lists));
      __syncthreads();
      for (int l = tid; l < lists; l += kBeamThreads) {
        const int i = l / parts, r = r0 + i;
        const bool ended = a.done && a.done[r];
        int j = at[l], stop = min((int)len[l], j + quota);
        for (; j < stop; ++j) {
          const u64 c = ended ? 0 : p.list[((int64_t)r * parts + l % parts) * k + j];
          const u64 score = order64(ended ? base[i] : base[i] + (double)logit_of((uint32_t)(c >> 32)));
          const u64 who = ((u64)r << 32) | (unsigned)(ended ? 0 : column_of(c) + 1);
          if (n == k && !(score > low_key || (score == low_key && who < low_pay))) {
            len[l] = 0;
            break;
          }
          const int to = atomicAdd(&s_n, 1);
          key[to] = score;
          pay[to] = who;
        }
        at[l] = j;
        if (j < len[l]) s_more = 1;
      }
      __syncthreads();
      const int came = s_n;
      const bool more = s_more;
      if (came > n) {
        int size = 64;
        while (size < came) size <<= 1;
        for (int i = came + tid; i < size; i += kBeamThreads) key[i] = 0, pay[i] = ~0ull;
        sort_desc<true>(key, pay, size);
        n = min(came, k);
      }
      if (!more) break;
    }
  }
  __syncthreads();

  if (tid == 0) a.count[b] = n;
  for (int i = tid; i < k; i += kBeamThreads) {
    const int64_t o = (int64_t)b * k + i;
    const int r = i < n ? (int)(pay[i] >> 32) : -1, col = i < n ? (int)(unsigned)pay[i] - 1 : -1;
    const u64 u = i < n ? key[i] : 0;
    a.parent[o] = r < 0 ? -1 : a.row_id ? a.row_id[r] : r;
    a.token[o] = col < 0 ? -1 : a.token_base + col;
    a.score_out[o] = r < 0 ? -INFINITY : (float)__longlong_as_double((long long)(u >> 63 ? u ^ (1ull << 63) : ~u));
  }
  if (!a.paths) return;
  for (int i = tid; i < k * a.max_path; i += kBeamThreads) {
    const int j = i / a.max_path, s = i % a.max_path;
    int v = -1;
    if (j < n) {
      const int r = (int)(pay[j] >> 32), col = (int)(unsigned)pay[j] - 1, id = a.row_id ? a.row_id[r] : r;
      const bool known = (unsigned)id < (unsigned)a.n_paths;
      const int held = known ? min(max(a.path_len[id], 0), a.max_path) : 0;
      if (s < held) v = a.paths[(int64_t)id * a.max_path + s];
      else if (s == held && col >= 0) v = a.token_base + col;
      if (s == 0) a.path_len_out[(int64_t)b * k + j] = held + (col >= 0 && held < a.max_path);
    } else if (s == 0) {
      a.path_len_out[(int64_t)b * k + j] = 0;
    }
    a.paths_out[((int64_t)b * k + j) * a.max_path + s] = v;
  }
}

static atspeed_status check_beam(const atspeed_beam_select_args& a) {
  if (a.dtype != ATSPEED_FP32 && a.dtype != ATSPEED_BF16) return fail(ATSPEED_E_INVALID, "dtype");
  if (a.B < 1 || a.B > kMaxRequests) return fail(ATSPEED_E_INVALID, "B must be 1..1024");
  if (a.n_rows < 0) return fail(ATSPEED_E_INVALID, "n_rows must be >= 0");
  if (a.n_cols < 1 || a.n_cols > (1 << 20)) return fail(ATSPEED_E_INVALID, "n_cols must be 1..2^20");
  if (a.k < 1 || a.k > kMaxBeams) return fail(ATSPEED_E_INVALID, "k must be 1..256");
  if (a.logits_stride < a.n_cols && a.n_rows > 1) return fail(ATSPEED_E_SHAPE, "a row stride is below n_cols");
  if (!a.row_off || !a.count || !a.parent || !a.token || !a.score_out || (a.n_rows > 0 && !a.logits))
    return fail(ATSPEED_E_INVALID, "beam select: null pointer");
  if ((a.paths != nullptr) != (a.path_len != nullptr)) return fail(ATSPEED_E_INVALID, "paths and path_len go together");
  if (a.paths) {
    if (a.n_paths < 1 || a.max_path < 1 || a.max_path > (1 << 16))
      return fail(ATSPEED_E_INVALID, "n_paths must be >= 1 and max_path 1..2^16");
    if (!a.paths_out || !a.path_len_out) return fail(ATSPEED_E_INVALID, "paths without their outputs");
  }
  const void* in[] = {a.logits, a.row_off, a.score, a.done, a.row_id, a.paths, a.path_len};
  const void* out[] = {a.count, a.parent, a.token, a.score_out, a.paths ? a.paths_out : nullptr,
                       a.paths ? a.path_len_out : nullptr};
  for (const void* i : in)
    for (const void* o : out)
      if (i && i == o) return fail(ATSPEED_E_INVALID, "beam select: an output is one of the inputs");
  if ((int64_t)a.k * a.max_path >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "beam select: k x max_path");
  return ATSPEED_OK;
}

// Parts of a row: enough workgroups for the card, of four tiles (one a wave) at least.
static void cut_rows(const atspeed_beam_select_args& a, BeamArgs& p) {
  const int tiles = (a.n_cols + kTile - 1) / kTile, rows = std::max(a.n_rows, 1);
  const int most = std::max(1, tiles / kBeamWaves), want = (1024 + rows - 1) / rows;
  p.tiles = (tiles + std::min(most, want) - 1) / std::min(most, want);
  p.parts = (tiles + p.tiles - 1) / p.tiles;
}

static size_t lay_out(BeamArgs& p, char* base) {
  const size_t lists = (size_t)std::max(p.a.n_rows, 1) * p.parts;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* q = base ? base + at : nullptr;
    at += (bytes + 255) & ~(size_t)255;
    return q;
  };
  p.list = (u64*)take(lists * p.a.k * 8);
  p.stat = (double2*)take(lists * 16);
  p.len = (int*)take(lists * 4);
  return at;
}

template <class T, int P>
static void launch_rows(const BeamArgs& p, unsigned grid, hipStream_t st) {
  int sorted = 64;
  while (sorted < kBeamWaves * p.a.k) sorted <<= 1;
  const size_t lds = ((size_t)kBeamWaves * Pool<P>::CAP + sorted) * 8;
  if (p.a.log_probs)
    hipLaunchKernelGGL((beam_rows_kernel<T, P, true>), dim3(grid), dim3(kBeamThreads), lds, st, p);
  else
    hipLaunchKernelGGL((beam_rows_kernel<T, P, false>), dim3(grid), dim3(kBeamThreads), lds, st, p);
}
// A pool holds k columns and 64 more at least.
template <class T>
static void launch_pool(const BeamArgs& p, unsigned grid, hipStream_t st) {
  if (p.a.k <= 64) launch_rows<T, 2>(p, grid, st);
  else if (p.a.k <= 192) launch_rows<T, 4>(p, grid, st);
  else launch_rows<T, 6>(p, grid, st);
}

}  // namespace atspeed

using namespace atspeed;

extern "C" {

atspeed_status atspeed_beam_select_workspace_bytes(const atspeed_beam_select_args* args, size_t* bytes) {
  if (!args || !bytes) return fail(ATSPEED_E_INVALID, "args or bytes is null");
  ST_TRY(check_beam(*args));
  BeamArgs p{};
  p.a = *args;
  cut_rows(*args, p);
  *bytes = lay_out(p, nullptr);
  return ATSPEED_OK;
}

atspeed_status atspeed_beam_select(const atspeed_beam_select_args* args, void* workspace, size_t ws_bytes, void* stream) {
  if (!args) return fail(ATSPEED_E_INVALID, "args is null");
  ST_TRY(check_beam(*args));
  BeamArgs p{};
  p.a = *args;
  cut_rows(*args, p);
  const long long groups = (long long)args->n_rows * p.parts;
  if (groups > kMaxGroups) return fail(ATSPEED_E_SHAPE, "beam select: too many rows x columns");
  const size_t need = lay_out(p, nullptr);
  if (!workspace || !aligned16(workspace) || ws_bytes < need)
    return fail(ATSPEED_E_WORKSPACE, "beam select: workspace is too small or not 16-byte aligned");
  lay_out(p, (char*)workspace);
  const hipStream_t st = (hipStream_t)stream;
  if (groups > 0) {
    if (args->dtype == ATSPEED_BF16) launch_pool<bf16_t>(p, (unsigned)groups, st);
    else launch_pool<float>(p, (unsigned)groups, st);
    HIP_TRY(hipGetLastError());
  }
  hipLaunchKernelGGL(beam_join_kernel, dim3(args->B), dim3(kBeamThreads), 0, st, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}

}  // extern "C"
