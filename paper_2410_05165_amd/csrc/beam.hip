// The k best continuations of each request's beams over the vocabulary
// (atspeed_beam_select).
//
// Within a row the order is that of the logits, so a first kernel reads every logit once
// and leaves the normaliser's sum and the k best logits of each part of a row; a second one
// ranks a request's lists by (score[r] - log sum) + (logit - largest).  In that order: a score is
// lost beside a logit of 3e38, and a row masked by such a number would rank as if it had none.
//
// Scores of different beams are compared, so their normalisers must not move them past each
// other.  They are taken in 64 bits, the exponentials to 2.4e-10: fp32 ones, off by 1e-7, would
// leave to chance which of two candidates that close comes first.  A 64-bit vector instruction
// takes the time of a 32-bit one here (1.8 ns a wave and SIMD), an fp32 exponential that of two.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "paged.h"
#include "wave.h"

namespace atspeed {

constexpr int kBeamThreads = 256, kBeamWaves = kBeamThreads / 64;
constexpr int kLane = 16;              // columns of a lane in a tile
constexpr int kTile = 64 * kLane;      // columns of a tile, which a wave takes at once
constexpr int kMaxBeams = 256;         // k
constexpr int kSlots = 4096;           // waves on the card at once, four a SIMD (five with small pools)

// Logits (no NaN) to whole numbers of the same order and as many bits, -0 as 0; and back.
template <class T>
__device__ __forceinline__ uint32_t order_of(float x) { return float_order_key(x + 0.f) >> (32 - 8 * sizeof(T)); }
template <class T>
__device__ __forceinline__ float logit_of(uint32_t order) {
  const uint32_t key = order << (32 - 8 * sizeof(T));
  const uint32_t bits = key & 0x80000000u ? key ^ 0x80000000u : ~key;
  return __uint_as_float(sizeof(T) == 2 ? bits & 0xffff0000u : bits);
}
// A column's place among its row's, by the logit, then the lower column: the logit's order over
// 0xffffffff - column.
__device__ __forceinline__ int column_of(u64 key) { return (int)(0xffffffffu - (unsigned)key); }
__device__ __forceinline__ u64 order64(double x) {
  const u64 u = (u64)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | (1ull << 63);
}
__device__ __forceinline__ double score_of(u64 u) {
  return __longlong_as_double((long long)(u >> 63 ? u ^ (1ull << 63) : ~u));
}

// A lane's 16 columns of a tile: 16-byte loads of consecutive lanes, wherever the row begins.
template <class T>
struct Tile {
  static constexpr int VEC = 16 / sizeof(T);
  static constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80u : 0xff800000u;   // -infinity
  u32x4_t raw[kLane / VEC];

  static __device__ __forceinline__ int column(int lane, int e) { return (e / VEC) * (64 * VEC) + lane * VEC + e % VEC; }
  // Columns c0 .. c0 + kTile - 1 of a row that has them.
  __device__ __forceinline__ void load(const T* row, int c0, int lane) {
#pragma unroll
    for (int v = 0; v < kLane / VEC; ++v) raw[v] = *reinterpret_cast<const u32x4_any_t*>(row + c0 + (v * 64 + lane) * VEC);
  }
  // All columns of a row of less than a tile, -infinity behind them.
  __device__ __forceinline__ void load_short(const T* row, int n_cols, int lane) {
#pragma unroll
    for (int v = 0; v < kLane / VEC; ++v)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
          const int c = column(lane, v * VEC + w * (VEC / 4) + i);
          uint32_t x = kNone;
          if (c < n_cols) x = VEC == 4 ? reinterpret_cast<const uint32_t*>(row)[c] : reinterpret_cast<const uint16_t*>(row)[c];
          word |= x << (16 * i);
        }
        raw[v][w] = word;
      }
  }
  // -infinity in the first n columns.
  __device__ __forceinline__ void drop(int n, int lane) {
    const int at = lane * VEC;
#pragma unroll
    for (int v = 0; v < kLane / VEC; ++v)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int c = v * 64 * VEC + w * (VEC / 4);
        if (VEC == 4) {
          raw[v][w] = at < n - c ? kNone : raw[v][w];
        } else {
          const uint32_t lo = at < n - c ? kNone : raw[v][w] & 0xffffu;
          raw[v][w] = lo | (at < n - c - 1 ? kNone << 16 : raw[v][w] & 0xffff0000u);
        }
      }
  }
  // What is computed from the tile behind this is not computed before.
  __device__ __forceinline__ void here() {
#pragma unroll
    for (int v = 0; v < kLane / VEC; ++v) asm volatile("" : "+v"(raw[v]));
  }
  __device__ __forceinline__ float operator[](int e) const {
    const uint32_t w = raw[e / VEC][e % VEC / (VEC / 4)];
    return __uint_as_float(VEC == 4 ? w : e & 1 ? w & 0xffff0000u : w << 16);
  }
};

// Largest t such that at least k of the wave's N numbers a lane are >= t, from bits
// 2 from + 1 and 2 from down to those of `to`; the bits above are t's.  Two bits a step: a
// step's length is that of one chain vector compare, count, scalar compare.
template <int N>
__device__ __forceinline__ uint32_t kth_largest(uint32_t (&x)[N], int k, uint32_t t, int from, int to) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));   // as numbers, not as the conditions they come from
#pragma unroll 1
  for (int step = from; step >= to; --step) {
    const uint32_t one = 1u << (2 * step);
    int n[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int d = 0; d < 3; ++d) n[d] += __popcll(__ballot(x[i] >= t + (d + 1) * one));
    t += n[2] >= k ? 3 * one : n[1] >= k ? 2 * one : n[0] >= k ? one : 0;
  }
  return t;
}

// Lanes before this one with a set bit.
__device__ __forceinline__ int lanes_before(u64 bits) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
}

// A wave's best columns so far, up to P * 64 of them in LDS, in no order: the logit's bits
// over the column's, which few instructions put there; their keys are made when they are read.
template <class T, int P>
struct Pool {
  static constexpr int CAP = P * 64;
  u64* at;
  int n;
  u64 least;    // columns at or below it are not among the wave's k best
  float bound;  // columns of the tiles to come are above it, or not above `least`

  static __device__ __forceinline__ u64 key_of(u64 x) {
    return (u64)order_of<T>(__uint_as_float((uint32_t)(x >> 32))) << 32 | (0xffffffffu - (uint32_t)x);
  }
  // Keeps the k best; high: no column lies above it.
  __device__ __forceinline__ void cut(int k, uint32_t high, int lane) {
    u64 own[P], x[P];
    uint32_t hi[P];
    wave_sync();
#pragma unroll
    for (int i = 0; i < P; ++i) {
      own[i] = at[i * 64 + lane];
      x[i] = i * 64 + lane < n ? key_of(own[i]) : 0;
      hi[i] = (uint32_t)(x[i] >> 32);
    }
    // the bits that the bounds have in common are the k-th's, too
    const uint32_t differ = (uint32_t)(least >> 32) ^ high;
    const int from = differ ? (31 - __builtin_clz(differ)) / 2 : -1;
    const uint32_t t = kth_largest<P>(hi, k, from == 15 ? 0u : high >> (2 * from + 2) << (2 * from + 2), from, 0);
    int above = 0, level = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      above += __popcll(__ballot(hi[i] > t));
      level += __popcll(__ballot(hi[i] == t));
    }
    u64 first = (u64)t << 32;
    if (above + level > k) {                    // equal logits: the lowest columns
      uint32_t lo[P];
#pragma unroll
      for (int i = 0; i < P; ++i) lo[i] = hi[i] == t ? (uint32_t)x[i] : 0;
      first |= kth_largest<P>(lo, k - above, 0u, 15, 0);
    }
    wave_sync();
    n = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const bool in = x[i] >= first && x[i];
      const u64 all = __ballot(in);
      if (in) at[n + lanes_before(all)] = own[i];
      n += __popcll(all);
    }
    n = min(n, k);                              // rows with NaN: any k
    least = max(least, first - 1);
    bound = logit_of<T>(t);                     // an equal logit further on has a higher column
    wave_sync();
  }

  // Takes in a tile's columns above the bound (c: the lane's first one); k and 64 more have room.
  __device__ __forceinline__ void add(Tile<T> x, int c, int k, uint32_t high, int lane) {
    for (;;) {
      x.here();
      u64 in[kLane];
      int all = 0;
#pragma unroll
      for (int e = 0; e < kLane; ++e) {
        in[e] = __ballot(x[e] > bound);
        all += __popcll(in[e]);
      }
      if (n + all <= CAP) {
#pragma unroll
        for (int e = 0; e < kLane; ++e) {
          if (!in[e]) continue;
          if (in[e] >> lane & 1)
            at[n + lanes_before(in[e])] = (u64)__float_as_uint(x[e]) << 32 | (uint32_t)(c + Tile<T>::column(0, e));
          n += __popcll(in[e]);
        }
        return;
      }
      if (n <= k) break;
      cut(k, high, lane);                       // few pass the bound that it leaves
    }
    // more than there is room for: a column a lane at a time, against the bound of the last cut
    for (int e = 0; e < kLane; ++e) {
      x.here();
      float z = -INFINITY;
      int col = 0;
#pragma unroll
      for (int i = 0; i < kLane; ++i)
        if (e == i) {
          z = x[i];
          col = c + Tile<T>::column(0, i);
        }
      const u64 is = (u64)__float_as_uint(z) << 32 | (uint32_t)col, key = z > -INFINITY ? key_of(is) : 0;
      u64 lanes = __ballot(key > least);
      if (n + __popcll(lanes) > CAP) {
        cut(k, high, lane);
        lanes = __ballot(key > least);
      }
      if (key > least) at[n + lanes_before(lanes)] = is;
      n += __popcll(lanes);
    }
  }
};

// sum += e^(x[e] - top) over a lane's columns, four chains at a time.  Differences below kLeast,
// those of -infinity among them, are held at it, which leaves nothing; in 64 bits, since fp32 has
// no numbers just below a `top` of 2^34.
template <class T>
__device__ __forceinline__ void add_exps(double& sum, float top, const Tile<T>& x) {
#pragma unroll
  for (int e = 0; e < kLane; e += 4) {
    double d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = fmax((double)x[e + i] - (double)top, (double)kLeast);
    exp_64(d);
    sum += (d[0] + d[1]) + (d[2] + d[3]);
  }
}

struct BeamArgs {
  atspeed_beam_select_args a;
  u64* list;        // [lists, k] the best columns, best first: a list a row, from some row on `parts` a row
  double2* stat;    // [lists] largest logit and sum of exponentials; NaN: the row has no candidates
  int* len;         // [lists]
  int whole, slack, parts, tiles, shift;   // rows below about `whole` have one list; tiles of a part; parts <= 1 << shift

  // The first list of row r where rows are cut from `from` on.
  __host__ __device__ int64_t list_of(int r, int from) const { return r < from ? r : from + (int64_t)(r - from) * parts; }
  __host__ __device__ int64_t most_lists(int rows) const { return list_of(rows, whole - slack); }
};

// The row from which on rows are cut: where the request that row `whole` lies in begins, or ends
// where it begins more than `slack` rows before.  A sum by parts differs from one of the whole row
// in its last bits, and rows of one request that are alike rank by their numbers: all of a
// request's rows are taken in one way.  The whole wave's call.
__device__ __forceinline__ int first_cut(const BeamArgs& p, int lane) {
  if (!p.slack) return p.whole;
  const int B = p.a.B, step = (B + 64) / 64, n_rows = p.a.n_rows;
  const u64 far = __ballot(p.a.row_off[min((lane + 1) * step - 1, B)] >= p.whole);
  if (!far) return n_rows;
  const int at = min((int)__builtin_ctzll(far) * step + min(lane, step - 1), B);
  const int end = p.a.row_off[at], begin = p.a.row_off[max(at - 1, 0)];
  const int first = __builtin_ctzll(__ballot(end >= p.whole));
  const int e = __builtin_amdgcn_readlane(end, first), b = __builtin_amdgcn_readlane(begin, first);
  return e > p.whole && b < p.whole && b >= p.whole - p.slack ? b : min(e, n_rows);
}

// A wave takes a part of a row by itself, tile by tile: the running maximum and 64-bit sum
// of its exponentials, and its k best columns behind a bound that rises with them.  No barrier,
// and the whole row where that fills the card: parts cost a pool and a first bound each.
// Bound by vector instructions, of which a tile's exponentials are half and the selection,
// which grows with k, a quarter: 5,661 rows of 33,024 bf16 columns with 50 beams each 180 to 186 us
// (374 MB, 2.0 TB/s; the call with 10 beams 153), 287 rows with 10 17.6.  A workgroup per row with
// a sorted pool took 393 and 39; without exponentials or selection it was 80.
template <class T, int P, bool PROBS>
__global__ void __launch_bounds__(kBeamThreads) beam_rows_kernel(BeamArgs p) {
  __shared__ u64 keys[kBeamWaves * P * 64];
  const atspeed_beam_select_args& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q = blockIdx.x * kBeamWaves + wave, from = q < p.whole - p.slack ? p.whole : first_cut(p, lane);
  const int cut = max(q - from, 0), part = cut % p.parts, r = min(q, from) + cut / p.parts;
  if (r >= a.n_rows) return;
  const int k = a.k, n_cols = a.n_cols;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.logits_stride;
  const uint32_t lowest = order_of<T>(-INFINITY);
  Pool<T, P> pool{keys + wave * P * 64, 0, (u64)lowest << 32 | 0xffffffffu, -INFINITY};
  float top = -INFINITY;
  double sum = 0.0;
  uint32_t high = 0;

  const int tiles = (n_cols + kTile - 1) / kTile, begin = part * p.tiles, end = q < from ? tiles : min(begin + p.tiles, tiles);
  // the last tile of a row ends with it and drops what the one before had
  const int last = n_cols - kTile;
  Tile<T> x, next;
  if (last < 0) next.load_short(row, n_cols, lane);
  else next.load(row, min(begin * kTile, last), lane);
  if (r >= a.row_off[a.B] || (a.done && a.done[r])) return;
  for (int tile = begin; tile < end; ++tile) {
    const int c0 = last < 0 ? 0 : min(tile * kTile, last);
    x = next;
    if (tile + 1 < end) next.load(row, min(c0 + kTile, last), lane);
    if (c0 != tile * kTile) x.drop(tile * kTile - c0, lane);
    float most[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) most[g] = max_nan(max_nan(x[4 * g], x[4 * g + 1]), max_nan(x[4 * g + 2], x[4 * g + 3]));
    const float mine = max_nan(max_nan(most[0], most[1]), max_nan(most[2], most[3]));
    if (__any(!(mine <= top))) {
      const float now = wave_max_nan(max_nan(mine, top));
      if (!PROBS && top > -INFINITY) sum *= exp_below(top, now);
      top = now;
      high = __builtin_amdgcn_readfirstlane(order_of<T>(top));
    }
    if (!PROBS && top > -INFINITY) add_exps(sum, top, x);
    if (tile == begin) {
      // k of 256 groups' largest are at or above the k-th of them; its upper 16 bits
      uint32_t o[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) o[g] = order_of<T>(most[g]);
      constexpr int STEPS = 4 * sizeof(T);
      const uint32_t t = kth_largest<4>(o, k, 0u, STEPS - 1, STEPS - 8);
      if (t > lowest + 1) {
        pool.least = ((u64)t << 32) - 1;
        pool.bound = logit_of<T>(t - (t == order_of<T>(0.f) ? 2 : 1));   // -0 is no number of its own
      }
    }
    if (__any(mine > pool.bound)) pool.add(x, c0 + Tile<T>::column(lane, 0), k, high, lane);
  }
  if (P > 2 && pool.n > k) pool.cut(k, high, lane);
  sum = wave_sum(sum);
  // in order: a column's place is the number of better ones
  wave_sync();
  const int n = pool.n, n8 = (n + 7) & ~7;
  u64 own[P];
  int place[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    own[i] = i * 64 + lane < n ? pool.key_of(pool.at[i * 64 + lane]) : 0;
    place[i] = 0;
    pool.at[i * 64 + lane] = own[i];
  }
  wave_sync();
  for (int j = 0; j < n8; j += 8) {
    u64 other[8];
#pragma unroll
    for (int o = 0; o < 8; ++o) other[o] = pool.at[j + o];
#pragma unroll
    for (int o = 0; o < 8; ++o)
#pragma unroll
      for (int i = 0; i < P; ++i) place[i] += other[o] > own[i];
  }
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (i * 64 + lane < n && place[i] < k) p.list[(int64_t)q * k + place[i]] = own[i];
  if (lane == 0) {
    p.stat[q] = {(double)top, top < INFINITY ? sum : NAN};
    p.len[q] = min(n, k);
  }
}

// ---------------------------------------------------------------- ranking a request's lists
// A workgroup a request.  Rounds: every list that may still count gives its next few
// entries, as many as the workgroup holds; the k-th of the threads' largest is a bound that
// few more than k of them pass; these are ranked, the k best stay.  A list is left once its
// last entry is behind them.  Mostly one round or two.  Bound by latency, a chain of loads and
// barriers: ten lists of ten 7.4 us, 32 requests of 99 lists of ten 10.9, 128 of 45
// rows, a third of them in three parts, 20.
constexpr int kEach = 4, kJoinLists = 1024;
constexpr short kItself = -1;              // length of the list of a row that has ended

// A candidate: its score's order (0: none), and row << 32 | column + 1.
__device__ __forceinline__ bool ahead_of(u64 key, u64 who, u64 than_key, u64 than_who) {
  return (key > than_key) | ((key == than_key) & (who < than_who));
}

constexpr int kBins = 1024;
// The bin of a distance: its exponent and four bits of it, from 2^-24 to 2^40.
__device__ __forceinline__ uint32_t bin_of(double d) {
  const int b = (int)(__float_as_uint((float)d) >> 19) - ((127 - 24) << 4);
  return (uint32_t)min(max(b, 0), kBins - 1);
}

template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) beam_join_kernel(BeamArgs p) {
  constexpr int WAVES = THREADS / 64, ROUND = THREADS * kEach, POOL = 2 * ROUND;   // a power of two
  extern __shared__ u64 key[];                     // [POOL]
  u64* const who_of = key + POOL;                  // [POOL]
  double* const base = (double*)(who_of + POOL);   // [kJoinLists] of a row: score - log sum,
  float* const largest_of = (float*)(base + kJoinLists);               // [kJoinLists] and what its logits are less
  unsigned short* const open = (unsigned short*)(largest_of + kJoinLists);   // [kJoinLists]
  short* const at = (short*)(open + kJoinLists);   // [kJoinLists]
  short* const len = at + kJoinLists;              // [kJoinLists]
  __shared__ u64 best_key[kMaxBeams], best_who[kMaxBeams], most[WAVES];
  __shared__ int bin[kBins], rank[THREADS], s_n, s_open[2];
  const atspeed_beam_select_args& a = p.a;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.k, shift = p.shift;
  const int r1 = min(min(a.row_off[b + 1], a.row_off[a.B]), a.n_rows);   // rows that the first kernel read
  const int group = kJoinLists >> shift;           // lists: row << shift | part
  const int cut_from = first_cut(p, lane);
  int n = 0;                                       // best_key[0 .. n) are the best so far, in order
  if (tid < 2) s_open[tid] = 0;
  for (int r0 = max(a.row_off[b], 0); r0 < r1; r0 += group) {
    const int rows = min(group, r1 - r0), lists = rows << shift;
    __syncthreads();
    // a group of lanes a row, a lane a part
    const int wide = min(shift, 6), lanes = 1 << wide;
    for (int i0 = 0; i0 < rows; i0 += THREADS >> wide) {
      const int i = i0 + (tid >> wide), r = min(r0 + i, r1 - 1), l = tid & (lanes - 1);
      const double score = a.score ? (double)a.score[r] : 0.0;
      const bool ended = a.done && a.done[r];
      const int parts = r < cut_from ? 1 : p.parts;
      double all = -INFINITY, total = 0.0;
      for (int q = l; q < 1 << shift; q += lanes) {
        // asked for before it is known whether the row has ended, and then left alone
        double2 st = {-INFINITY, 0.0};
        int length = 0;
        if (q < parts) {
          st = p.stat[p.list_of(r, cut_from) + q];
          length = p.len[p.list_of(r, cut_from) + q];
        }
        if (ended) st = {-INFINITY, 0.0};
        if (i < rows) {
          at[i << shift | q] = 0;
          len[i << shift | q] = !ended ? (short)length : q == 0 ? kItself : 0;
        }
        // NaN stays; a part whose largest logit is -infinity has nothing to add
        const double now = st.x > all ? st.x : all, add = st.x > -INFINITY ? st.y : st.x == -INFINITY ? 0.0 : NAN;
        total = q == l || a.log_probs ? total + add : total * exp_below(all, now) + add * exp_below(st.x, now);
        all = now;
      }
      double most_of = all;
      for (int o = 1; o < lanes; o <<= 1) most_of = fmax(most_of, __shfl_xor(most_of, o));
      if (!a.log_probs && all > -INFINITY) total *= exp_below(all, most_of);
      all = most_of;
      for (int o = 1; o < lanes; o <<= 1) total += __shfl_xor(total, o);
      bool none = !(fabs(score) < INFINITY) || !(total == total);
      double x = score;
      if (!ended && !a.log_probs) {
        x = score - log(total);                    // without columns: infinite
        none = none || !(fabs(x) < INFINITY);
      }
      if (i < rows && l == 0) {
        base[i] = x;
        largest_of[i] = a.log_probs ? 0.f : (float)all;
      }
      if (i < rows && none)
        for (int q = l; q < 1 << shift; q += lanes) len[i << shift | q] = 0;
    }
    for (int round = 0;; round ^= 1) {
      // the lists that are left
      __syncthreads();
      for (int l0 = 0; l0 < lists; l0 += THREADS) {
        const int l = l0 + tid, length = l < lists ? len[l] : 0;
        const bool is = l < lists && at[l] < (length == kItself ? 1 : length);
        const u64 all = __ballot(is);
        int to = 0;
        if (lane == 0 && all) to = atomicAdd(&s_open[round], __popcll(all));
        to = __builtin_amdgcn_readfirstlane(to) + lanes_before(all);
        if (is) open[to] = (unsigned short)l;
      }
      if (tid == 0) s_n = 0;
      __syncthreads();
      const int n_open = s_open[round];
      if (tid == 0) s_open[round ^ 1] = 0;
      if (!n_open) break;
      // a power of two of each, k at most
      int depth = 31 - __builtin_clz((unsigned)(ROUND / n_open));
      while (depth > 0 && 1 << (depth - 1) >= k) --depth;

      // a thread's entries, and its place among the best so far
      u64 mine[kEach + 1], who[kEach + 1], largest = 0, listed[kEach];
      int from[kEach], next[kEach];                // next: where its list goes on, -1: it ends here, 0: not the last one taken
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int e = tid + i * THREADS, o = min(e >> depth, n_open - 1), l = open[o], d = e & ((1 << depth) - 1);
        const int j = at[l] + d, length = len[l], n_here = length == kItself ? 1 : length;
        const bool in = e >> depth < n_open && j < n_here;
        from[i] = in ? l : -1;
        next[i] = j + 1 >= n_here ? -1 : d + 1 == 1 << depth ? j + 1 : 0;
        listed[i] = in && length != kItself ? p.list[(p.list_of(r0 + (l >> shift), cut_from) + (l & ((1 << shift) - 1))) * k + j] : 0;
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int row = max(from[i], 0) >> shift;
        const double below = listed[i] ? (double)logit_of<T>((uint32_t)(listed[i] >> 32)) - (double)largest_of[row] : 0.0;   // a key is never 0
        mine[i] = from[i] >= 0 ? order64(base[row] + below) : 0;
        who[i] = (u64)(r0 + row) << 32 | (listed[i] ? column_of(listed[i]) + 1 : 0);
        largest = max(largest, mine[i]);
      }
      mine[kEach] = tid < n ? best_key[tid] : 0;
      who[kEach] = tid < n ? best_who[tid] : 0;
      largest = max(largest, mine[kEach]);
      // Few entries are all ranked.  Of many, those that are at or above the k-th of the threads'
      // largest, in bins of a sixteenth of their distance to the best of all.
      uint32_t limit = kBins;
      double top = 0.0;
      if (n_open << depth > 64) {
        u64 high = largest;
        static_for<6>([&](auto s) { high = max(high, (u64)partner<s>((uint32_t)(high >> 32)) << 32 | partner<s>((uint32_t)high)); });
        if (lane == 0) most[wave] = high;
        for (int i = tid; i < kBins; i += THREADS) bin[i] = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) high = max(high, most[w]);
        top = score_of(high);
        if (largest) atomicAdd(&bin[bin_of(top - score_of(largest))], 1);
        __syncthreads();
        // a lane has sixteen bins: how many there are up to each
        int upto[kBins / 64];
#pragma unroll
        for (int i = 0; i < kBins / 64; ++i) upto[i] = bin[lane * (kBins / 64) + i] + (i ? upto[i - 1] : 0);
        const int before = wave_scan(upto[kBins / 64 - 1]) - upto[kBins / 64 - 1];
        int mine_limit = kBins;
#pragma unroll
        for (int i = kBins / 64 - 1; i >= 0; --i)
          if (before + upto[i] >= k) mine_limit = lane * (kBins / 64) + i;
        const u64 enough = __ballot(mine_limit < kBins);
        if (enough) limit = __builtin_amdgcn_readlane(mine_limit, __builtin_ctzll(enough));
      } else {
        __syncthreads();
      }
#pragma unroll
      for (int i = 0; i <= kEach; ++i)
        if (mine[i] && (limit == kBins || bin_of(top - score_of(mine[i])) <= limit)) {
          const int to = atomicAdd(&s_n, 1);
          key[to] = mine[i];
          who_of[to] = who[i];
        }
      rank[tid] = 0;
      __syncthreads();
      const int came = s_n;
      int size = 64;
      while (size < came) size <<= 1;
      if (size <= THREADS) {
        // A place is the number of better ones, counted by THREADS / size threads each; equal
        // scores, which are rare, are told apart behind that.
        const int per = max(size / (THREADS / size), 8);          // in eights: no entry belongs to two threads' parts
        const int e = tid & (size - 1), j0 = tid / size * per;
        if (tid >= came && tid < size) key[tid] = 0;
        __syncthreads();
        const u64 x = key[e];
        int before = 0, same = 0;
        for (int j = j0; j < min(came, j0 + per); j += 8) {
          u64 y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = key[(j + i) & (size - 1)];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            before += y[i] > x;
            same += y[i] == x;
          }
        }
        if (e < came && same > (e >= j0 && e < j0 + per))
          for (int j = j0; j < min(came, j0 + per); ++j) before += key[j] == x && who_of[j] < who_of[e];
        if (e < came && before) atomicAdd(&rank[e], before);
        __syncthreads();
        if (tid < came && rank[tid] < k) {
          best_key[rank[tid]] = key[tid];
          best_who[rank[tid]] = who_of[tid];
        }
      } else {
        for (int i = came + tid; i < size; i += THREADS) key[i] = 0, who_of[i] = ~0ull;
        for (int sorted = 2; sorted <= size; sorted <<= 1)
          for (int step = sorted >> 1; step; step >>= 1) {
            __syncthreads();
            for (int i = tid; i < size / 2; i += THREADS) {
              const int x = 2 * i - (i & (step - 1)), y = x + step;
              const u64 kx = key[x], ky = key[y], wx = who_of[x], wy = who_of[y];
              if (ahead_of(kx, wx, ky, wy) == ((x & sorted) != 0)) {
                key[x] = ky, key[y] = kx;
                who_of[x] = wy, who_of[y] = wx;
              }
            }
          }
        __syncthreads();
        if (tid < min(came, k)) {
          best_key[tid] = key[tid];
          best_who[tid] = who_of[tid];
        }
      }
      n = min(came, k);
      __syncthreads();
      // lists at their end or behind the k-th are done
      const u64 worst = n == k ? best_key[k - 1] : 0, worst_who = n == k ? best_who[k - 1] : ~0ull;
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (from[i] >= 0 && next[i]) {
          if (next[i] < 0 || ahead_of(worst, worst_who, mine[i], who[i])) len[from[i]] = 0;
          else at[from[i]] = (short)next[i];
        }
    }
  }
  __syncthreads();

  if (tid == 0) a.count[b] = n;
  int* const id_of = reinterpret_cast<int*>(key);   // [k] what parent names an entry's row by
  int* const held_of = id_of + kMaxBeams;           // [k] the length of its path
  for (int i = tid; i < k; i += THREADS) {
    const int64_t o = (int64_t)b * k + i;
    const int r = i < n ? (int)(best_who[i] >> 32) : -1, col = i < n ? (int)(unsigned)best_who[i] - 1 : -1;
    const int id = r < 0 ? -1 : a.row_id ? a.row_id[r] : r;
    a.parent[o] = id;
    a.token[o] = col < 0 ? -1 : a.token_base + col;
    a.score_out[o] = r < 0 ? -INFINITY : (float)score_of(best_key[i]);
    if (a.paths) {
      const bool known = r >= 0 && (unsigned)id < (unsigned)a.n_paths;
      const int held = known ? min(max(a.path_len[id], 0), a.max_path) : 0;
      a.path_len_out[o] = held + (col >= 0 && held < a.max_path);
      id_of[i] = id;
      held_of[i] = held;
    }
  }
  if (!a.paths) return;
  __syncthreads();
  for (int i = tid; i < k * a.max_path; i += THREADS) {
    const int j = i / a.max_path, s = i % a.max_path, held = held_of[j];
    const int col = j < n ? (int)(unsigned)best_who[j] - 1 : -1;
    const int there = a.paths[s < held ? (int64_t)id_of[j] * a.max_path + s : 0];
    a.paths_out[((int64_t)b * k + j) * a.max_path + s] = s < held ? there : s == held && col >= 0 ? a.token_base + col : -1;
  }
}

template <class T, int THREADS>
static atspeed_status launch_join(const BeamArgs& p, hipStream_t st) {
  constexpr int lds = 2 * THREADS * kEach * 16 + kJoinLists * 18;
  if (lds > (64 << 10))
    HIP_TRY(hipFuncSetAttribute((const void*)beam_join_kernel<T, THREADS>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  hipLaunchKernelGGL((beam_join_kernel<T, THREADS>), dim3(p.a.B), dim3(THREADS), lds, st, p);
  HIP_TRY(hipGetLastError());
  return ATSPEED_OK;
}
template <class T>
static atspeed_status run_join(const BeamArgs& p, hipStream_t st) {
  // Few entries a request, or many requests: smaller workgroups, more of them on a CU (both
  // kernels, us, 256 threads and 1,024: 10 rows of 1,024 columns 13.0 and 15.9, 32 requests of 9
  // rows of 33,024 with 10 beams 27.2 and 28.4; but 128 of 45 rows with 50 189 and 187).
  const long long entries = p.most_lists(p.a.n_rows) * p.a.k;
  return p.a.B > 256 || entries <= 1024LL * p.a.B ? launch_join<T, 256>(p, st) : launch_join<T, 1024>(p, st);
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

// Parts of a row: a wave each, enough waves for the card, but not many more lists a request
// than one round of the second kernel takes in (64 rows of one request, 128 beams: parts of one
// tile 89 us, of two 56, of five 50; 287 rows of 32 requests: 7 parts 27.8, 11 26.5, 17 27.3).
// As many rows as fill the card whole are not cut; few waves behind them would leave it half
// empty, so that those rows are (both kernels, us, with them in 1 part, 2 and 3: 4,300 rows 159,
// 138 and 138, 5,661 187, 184 and 180; 7,000 215, 216 and 221, 8,100 239, 246 and 251; all of
// 5,661 rows in 2 was 4% slower).
static void cut_rows(const atspeed_beam_select_args& a, BeamArgs& p) {
  const int tiles = (a.n_cols + kTile - 1) / kTile, rows = std::max(a.n_rows, 1), beams = (rows + a.B - 1) / a.B;
  p.whole = rows / kSlots * kSlots;
  const int rest = std::max(rows - p.whole, 1), most = std::max(1, std::min(tiles, kJoinLists / 2 / beams));
  const int want = std::min(most, std::max(1, (kSlots + rest / 2) / rest));
  p.tiles = (tiles + want - 1) / want;
  p.parts = (tiles + p.tiles - 1) / p.tiles;
  while (1 << p.shift < p.parts) ++p.shift;
  // the cut moves to where a request begins: twice the requests' average is room for most
  if (p.whole && p.parts > 1) p.slack = std::min(2 * beams, p.whole);
}

static size_t lay_out(BeamArgs& p, char* base) {
  const size_t lists = p.most_lists(std::max(p.a.n_rows, 1));
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
  if (p.a.log_probs)
    hipLaunchKernelGGL((beam_rows_kernel<T, P, true>), dim3(grid), dim3(kBeamThreads), 0, st, p);
  else
    hipLaunchKernelGGL((beam_rows_kernel<T, P, false>), dim3(grid), dim3(kBeamThreads), 0, st, p);
}
// A pool holds k columns and 64 more at least, and better the k and those that pass the first
// bound in a tile, 1.1 k for small k, more for large: what has no room waits for a cut (both
// kernels, us, smaller pool and larger: 5,632 rows of 33,024 bf16 columns, k = 50, 178 and 191, 56
// 189 and 196, 64 204 and 201; 200 fp32 rows, 56 37 and 33, 110 47 and 43, 192 88 and 75).
template <class T>
static void launch_pool(const BeamArgs& p, unsigned grid, hipStream_t st) {
  if (p.a.k <= 56) launch_rows<T, 2>(p, grid, st);
  else if (p.a.k <= 104) launch_rows<T, 4>(p, grid, st);
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
  const long long groups = (p.most_lists(args->n_rows) + kBeamWaves - 1) / kBeamWaves;
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
  return args->dtype == ATSPEED_BF16 ? run_join<bf16_t>(p, st) : run_join<float>(p, st);
}

}  // extern "C"
