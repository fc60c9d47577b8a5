// Tree attention over a paged cache (atspeed_tree_attention):
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),  j the keys a row sees,
// in one pass over the keys with a running maximum m.  The rows of a request times the
// query heads of one key/value head are the queries of a matrix tile, so grouped heads
// read the cache once for the group.  Two kernels: up to 32 queries (single tokens,
// small trees), bound by the reads of the cache, and more, bound by the matrix and
// vector instructions and the latencies between them; long contexts are cut into pieces
// and their parts joined.  Measured (us; share of a 4.95 TB/s copy or of a 1,214 TFLOP/s
// product): 64 single tokens over up to 8,192 keys, 8 of 32 heads, 143 (99% of the copy);
// 60 nodes x 32 users over 144 keys, 32 heads, 33.7 (83%); trees of 4 users over up to
// 65,536 keys 144 (82%); 300 nodes x 128 users over 1,024 keys 1,431 (0.45 PFLOP/s of
// what the rows see); causal chunks of up to 1,024 x 16 users 127 (0.54 PFLOP/s).  The
// comparisons of tiles, pieces and loops below were measured with probabilities as one
// bf16 number (see Tile), which takes 4 to 20% less where many rows are bound by the
// matrix work.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "paged.h"
#include "wave.h"

namespace atspeed {

struct TreeAttnArgs {
  const char* q;
  int64_t q_row, q_head;       // bytes
  const char* k;
  const char* v;
  int64_t k_head, v_head;      // bytes
  // where a token's row starts, in units of `unit` bytes: page * *_page + token * *_token
  uint32_t k_page, k_token, v_page, v_token, unit;
  const int* table;
  const int* row_off;
  const int* ctx;
  const uint64_t* mask;
  char* out;
  int64_t o_row, o_head;       // bytes
  float* lse;
  int4* split;                 // [B] where a split request's parts are: first unit, parts, tiles
  float* part;                 // [units][KH][qb][d_head] unnormalised sums
  float2* part_ml;             // [units][KH][qb] running maximum and sum
  int B, n_rows, H, G, KH, max_pages, n_pool, max_new, words, shift, tail;
  int qtiles, qb;              // query tiles of a request at most, queries of a tile
  int units;                   // workgroups a key/value head if requests are split, else 0
  int cap;                     // keys a request can have: max_pages pages, at most 2^30
  uint32_t q_flip;             // sign bits of the queries' elements (negative scale)
  float scale;                 // |scale| log2(e)
};

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // a maximum moves when a score passes it by 2^8

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
typedef __attribute__((address_space(3))) void lds_void_t;

// New rows of request b, from row r0 on; none where its offsets are no rows of the call.
__device__ __forceinline__ int new_rows(const TreeAttnArgs& a, int b, int& r0) {
  const int begin = a.row_off[b], end = a.row_off[b + 1];
  const bool sane = begin >= 0 && begin < a.n_rows && end > begin;
  r0 = sane ? begin : 0;
  return sane ? end - begin : 0;
}

__device__ __forceinline__ int round_up64(int n) { return (n + 63) & ~63; }

// One workgroup's share: a request, a key/value head, a tile of its queries (row i, head
// h of the group: query i * G + h), a range of its keys.
struct Share {
  int kvh, r0, nq, q0, unit, nsplit;
  int ctx, kbeg, kend;   // context keys; this workgroup's keys
  int clear;             // from this key on some query may not see a key
  const int* table;

  // False where there is nothing to do.  CUT: the requests are cut into pieces (kernels of
  // their own: the registers of pick() cost the others 2 to 12%).
  template <bool CUT>
  __device__ __forceinline__ bool init(const TreeAttnArgs& a) {
    int b, qt, split, total;
    if constexpr (CUT) {
      if (!pick(a, b, qt, split, total)) return false;
      // one value a wave, as the compiler cannot tell
      for (int* x : {&b, &qt, &split, &total, &kvh, &unit, &nsplit, &r0, &nq, &ctx}) *x = __builtin_amdgcn_readfirstlane(*x);
    } else {
      // Workgroup L runs on XCD L % 8: the tiles of one pair stay on one XCD, whose L2
      // then holds the pair's keys; the pairs are dealt round-robin.
      const int L = blockIdx.x, pair = ((L >> 3) / a.qtiles) * 8 + (L & 7), z = (L >> 3) % a.qtiles;
      if (pair >= a.B * a.KH) return false;
      b = pair / a.KH;
      kvh = pair % a.KH;
      qt = a.mask ? z : a.qtiles - 1 - z;   // chains: the tiles with the most keys first
      split = unit = 0;
      nsplit = 1;
      total = request(a, b);
    }
    q0 = qt * a.qb;
    if (q0 >= nq) return false;
    const int chunk = round_up64((total + nsplit - 1) / nsplit);
    kbeg = split * chunk;
    kend = split + 1 < nsplit ? min(kbeg + chunk, total) : total;   // the last pieces may be empty
    if (!a.mask) kend = min(kend, ctx + (min(q0 + a.qb, nq) - 1) / a.G + 1);
    clear = a.mask ? ctx : ctx + q0 / a.G + 1;
    table = a.table + (int64_t)b * a.max_pages;
    return true;
  }
  // Keys of request b; sets r0, nq and ctx.
  __device__ __forceinline__ int request(const TreeAttnArgs& a, int b) {
    const int count = new_rows(a, b, r0);
    nq = min(min(count, a.n_rows - r0), a.max_new) * a.G;   // fits: n_rows x heads does
    return keys(a, b, count);
  }
  // The workgroup's piece where requests are split: all requests into pieces of about c
  // keys, c such that they are a.units at most for a key/value head.  With S = sum of
  // tiles x keys and N = sum of tiles the pieces are S / c at least and S / c + N at most,
  // and a.units >= 2 N: c = S / units is enlarged by eighths until they fit, 2 S / units
  // at most.  Every wave works it out from the requests' lengths, 64 requests at a time,
  // and takes the workgroup's place in the list of the pieces.
  __device__ __forceinline__ bool pick(const TreeAttnArgs& a, int& b, int& qt, int& split, int& total) {
    const int lane = threadIdx.x & 63;
    int len, tiles;
    auto load = [&](int i) {
      len = tiles = 0;
      if (i >= a.B) return;
      len = request(a, i);
      tiles = (nq + a.qb - 1) / a.qb;
    };
    const bool one = a.B <= 64;   // the lengths stay in registers
    float S = 0;
    for (int i0 = 0; i0 < a.B; i0 += 64) {
      load(i0 + lane);
      S += wave_scan((float)len * tiles);
    }
    // sums of 1,024 numbers in fp32: 1e-6 off at most
    const float c0 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, S), 63)) * 1.00001f / a.units;
    float per_key;
    int all;
    auto pieces = [&]() { return tiles * (1 + (int)((float)max(len - 1, 0) * per_key)); };
    for (int e = 8; e <= 16; ++e) {
      per_key = 1.f / fmaxf(c0 * e * 0.125f, 256.f);
      int n = 0;
      for (int i0 = 0; i0 < a.B; i0 += 64) {
        if (!one) load(i0 + lane);
        n += wave_scan(pieces());
      }
      all = __builtin_amdgcn_readlane(n, 63);
      if (all <= a.units) break;
    }
    // Workgroup L runs on XCD L % 8, which takes neighbours in the list: the tiles of a
    // piece, which read the same keys.
    all = min(all, a.units);
    const int L = blockIdx.x, per = (all * a.KH + 7) / 8, at = (L & 7) * per + (L >> 3);
    if ((L >> 3) >= per || at >= all * a.KH) return false;
    kvh = at / all;
    unit = at % all;
    int left = unit;
    for (int i0 = 0; i0 < a.B; i0 += 64) {
      if (!one) load(i0 + lane);
      const int n = pieces(), upto = wave_scan(n);
      const uint64_t past = __ballot(upto > left);
      if (past) {
        const int l = __ffsll((unsigned long long)past) - 1, t = __builtin_amdgcn_readlane(tiles, l);
        b = i0 + l;
        left -= __builtin_amdgcn_readlane(upto - n, l);
        total = __builtin_amdgcn_readlane(len, l);
        r0 = __builtin_amdgcn_readlane(r0, l);
        nq = __builtin_amdgcn_readlane(nq, l);
        ctx = __builtin_amdgcn_readlane(ctx, l);
        nsplit = __builtin_amdgcn_readlane(n, l) / t;
        split = left / t;
        qt = left % t;
        if (left == 0 && kvh == 0 && threadIdx.x == 0) a.split[b] = int4{unit, nsplit, t, 0};
        return true;
      }
      left -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
  }
  // Keys of request b with `count` new rows (none where ctx is negative); sets ctx.
  __device__ __forceinline__ int keys(const TreeAttnArgs& a, int b, int count) {
    const int c = a.ctx[b];
    ctx = min(max(c, 0), a.cap);
    const int64_t n = a.mask ? min((int64_t)count, (int64_t)a.words * 64) : (int64_t)count;
    return c < 0 ? 0 : (int)min(c + n, (int64_t)a.cap);
  }
  // Page of key k0 + lane for the first n lanes, -1 where the key is not there.
  __device__ __forceinline__ int page(const TreeAttnArgs& a, int k0, int n) const {
    const int lane = threadIdx.x & 63, key = k0 + lane;
    return lane < n && key < kend ? table[key >> a.shift] : -1;
  }
};

// Rows of keys and values of one tile: lane i holds key i's.  Where a key is not there, it
// holds the first key's that is (page 0's where none is): what lies elsewhere in the cache
// is not the request's, and values that are not finite there would cost it a search.
struct TileRows {
  uint32_t k, v;     // units
  uint64_t there;    // bit i: key i is there
  // all: the bits of a whole tile.
  __device__ __forceinline__ void set(const TreeAttnArgs& a, int k0, int page, uint64_t all) {
    const bool ok = (unsigned)page < (unsigned)a.n_pool;
    const uint32_t pg = ok ? page : 0, tok = (k0 + (threadIdx.x & 63)) & a.tail;
    k = pg * a.k_page + tok * a.k_token;
    v = pg * a.v_page + tok * a.v_token;
    there = __ballot(ok);
    if (there != 0 && there != all) {
      const int first = __ffsll((unsigned long long)there) - 1;
      const uint32_t k1 = __builtin_amdgcn_readlane(k, first), v1 = __builtin_amdgcn_readlane(v, first);
      k = ok ? k : k1;
      v = ok ? v : v1;
    }
  }
};

// The keys of a wave's or workgroup's tiles in which values were left out (Tile::finite).
struct Holes {
  int begin = 1 << 30, end = 0;
  __device__ __forceinline__ void add(bool any_of_wave, int k0, int keys) {
    if (!any_of_wave) return;
    begin = min(begin, k0);
    end = k0 + keys;
  }
  // Those of the four waves (waits for them).
  __device__ __forceinline__ bool join(int2 (&all)[4], int wave) {
    if (!__syncthreads_or(end != 0)) return false;
    if ((threadIdx.x & 63) == 0) all[wave] = int2{begin, end};
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      begin = min(begin, all[w].x);
      end = max(end, all[w].y);
    }
    return true;
  }
};

// The mask words that hold bits j0 .. j0 + 63 of a row, and those bits.  Context keys
// (j < 0) are always seen, bits past the words never.
struct MaskWords {
  uint64_t lo, hi;
  __device__ __forceinline__ void load(const uint64_t* words, int n, int j0) {
    const int w = j0 < 0 ? 0 : j0 >> 6;
    lo = j0 > -64 && w < n ? words[w] : 0ull;
    hi = j0 > 0 && (j0 & 63) && w + 1 < n ? words[w + 1] : 0ull;
  }
  __device__ __forceinline__ uint64_t bits(int j0) const {
    if (j0 <= -64) return ~0ull;
    if (j0 < 0) return (lo << -j0) | ((1ull << -j0) - 1);
    const int s = j0 & 63;
    return s ? (lo >> s) | (hi << (64 - s)) : lo;
  }
};
// Without a mask: the keys up to the row's own, at ctx + i.
__device__ __forceinline__ uint64_t chain_bits(int i, int j0) {
  const int n = i + 1 - j0;
  return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
}

// A wave's arithmetic on NQ blocks of 16 queries and a tile of KW keys whose K and V
// rows lie in LDS.  S^T = K Q^T (v_mfma 16x16, A = K rows, B = Q): lane l holds the
// scores of query l % 16 with keys 4g .. 4g + 3 (g = l / 16) of each 16-key block, which
// is the B operand of O^T = V^T P^T, so probabilities stay in registers.  bf16: V^T's
// fragments come from a transposing LDS read (4 keys x 16 dims per 16 lanes) and the 32
// keys of a step are ordered {4g .. 4g + 3, 16 + 4g .. 16 + 4g + 3} on both operands;
// fp32: MFMA e of a block takes keys {e, 4 + e, 8 + e, 12 + e}.  Softmax in fp32 with a
// running maximum that moves only when a query's score passes it by 2^8 (probabilities up to
// 2^8 keep their relative precision, and the exchange between the lanes of a query and
// the rescaling are rare); lsum is each lane's own part until the end.  bf16
// probabilities meet V as two bf16 numbers, the upper 16 bits and the rest rounded: off
// by 2^-15 of each at most, so that they are those of fp32 in a bf16 output, like in
// the attention of the context's own forwards.  As one bf16 they added a third to
// the output's error (0.0022 for 0.0017, relative norm) and saved half of this product:
// (us, so; as one) 300 nodes x 128 users 1,437; 1,211, causal chunks of up to 1,024 x 16
// users 124; 103, 4 trees over up to 65,536 keys 150; 135, smaller launches of many rows
// 4 to 16% more, single tokens and small trees 0 to 2%.
template <class T, int DH, int NQ, int KW>
struct Tile {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int ROWB = DH * (int)sizeof(T);   // bytes of a row
  static constexpr int CPR = ROWB / 16;              // 16-byte chunks of a row
  static constexpr int NKS = CPR / 4;                // chunk groups of a score
  static constexpr int NDB = DH / 16;                // 16-dim blocks of the output
  static constexpr int NKB = KW / 16;                // 16-key blocks of the tile
  static constexpr int BYTES = KW * ROWB;            // of K, and of V
  static constexpr uint64_t ALL = KW == 64 ? ~0ull : (1ull << KW) - 1;

  // Chunk swizzles: K fragments are read 16 rows at one chunk; V (bf16) 8 rows at one
  // 16-dim block (two chunks), (fp32) 4 rows, 4 apart, at one 16-dim block.
  static __device__ __forceinline__ int kswz(int key) { return BF ? key & (CPR - 1) : CPR >= 16 ? key & 15 : (key >> 1) & 7; }
  static __device__ __forceinline__ int vswz(int key) {
    return BF ? (DH == 128 ? key & 7 : (key >> 1) & 3) << 1 : ((key >> 2) & (NDB >= 4 ? 3 : 1)) << 2;
  }

  int g, ql;
  int qi[NQ], qhead[NQ];     // the lane's queries: new-row index, head
  int64_t qrow[NQ];
  bool qok[NQ];
  f32x4_t qf[NQ][NKS];
  f32x4_t o[NQ][NDB];
  float m[NQ], lsum[NQ];

  // first: the wave's first query.
  __device__ __forceinline__ void init(const TreeAttnArgs& a, const Share& s, int first) {
    const int lane = threadIdx.x & 63;
    g = lane >> 4;
    ql = lane & 15;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int c = first + n * 16 + ql;
      qok[n] = c < s.nq;
      const int cc = qok[n] ? c : s.nq - 1;
      qi[n] = cc / a.G;
      qrow[n] = s.r0 + qi[n];
      qhead[n] = s.kvh * a.G + cc % a.G;
      const char* p = a.q + qrow[n] * a.q_row + qhead[n] * a.q_head + g * 16;
#pragma unroll
      for (int k = 0; k < NKS; ++k) {
        u32x4_t w = *reinterpret_cast<const u32x4_t*>(p + k * 64);
        w ^= a.q_flip;
        qf[n][k] = __builtin_bit_cast(f32x4_t, w);
      }
      m[n] = -INFINITY;
      lsum[n] = 0.f;
#pragma unroll
      for (int d = 0; d < NDB; ++d) o[n][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }

  // bits: the keys each query sees, if not `full` (all of them).  between(k) runs after
  // the k-th chunk group of the scores, k = 0 .. NKS - 1.  NB: the blocks of queries that
  // there are.
  template <int NB, class F>
  __device__ __forceinline__ void step(const TreeAttnArgs& a, const char* ks, const char* vs, bool full,
                                       const uint64_t (&bits)[NQ], F&& between) {
    f32x4_t sc[NB][NKB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) sc[n][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NKS; ++k) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) {
        const int key = kb * 16 + ql;
        const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(ks + key * ROWB + ((k * 4 + g) ^ kswz(key)) * 16);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if constexpr (BF) {
            sc[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf),
                                                                 __builtin_bit_cast(bf16x8_t, qf[n][k]), sc[n][kb], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[n][kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[n][k][e], sc[n][kb], 0, 0, 0);
          }
        }
      }
      between(k);
    }
    if (!full) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const uint64_t mine = bits[n] >> (g * 4);
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {   // a set bit keeps the score, a clear one makes it -inf
            const uint32_t half = (uint32_t)(kb < 2 ? mine : mine >> 32);
            const uint32_t keep = (uint32_t)((int32_t)(half << (31 - (kb & 1) * 16 - i)) >> 31);
            const uint32_t x = __float_as_uint(sc[n][kb][i]);
            sc[n][kb][i] = __uint_as_float((x & keep) | (0xff800000u & ~keep));
          }
      }
    }
    float mx[NB];
    bool moved = false;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      float x = sc[n][0][0];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) x = fmaxf(x, sc[n][kb][i]);
      mx[n] = x * a.scale;
      moved |= mx[n] > m[n] + kSlack;
    }
    if (__any(moved)) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float x = fmaxf(mx[n], __shfl_xor(mx[n], 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        // a query's own scores alone move its maximum, and with it its roundings
        const float mnew = x > m[n] + kSlack ? x : m[n];
        const float alpha = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - mnew);
        m[n] = mnew;
        lsum[n] *= alpha;
#pragma unroll
        for (int d = 0; d < NDB; ++d) o[n][d] *= alpha;
      }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const float ref = m[n] != -INFINITY ? m[n] : 0.f;   // a query that has seen nothing yet
      float ps = 0.f;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][kb][i], a.scale, -ref));
          sc[n][kb][i] = p;
          ps += p;
        }
      lsum[n] += ps;
    }
    if constexpr (BF) {
#pragma unroll
      for (int kk = 0; kk < KW / 32; ++kk) {
        bf16x8_t ph[NB], pl[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) {   // the upper 16 bits, and what they leave
            const float p = sc[n][2 * kk + i / 4][i % 4];
            const uint32_t bits = __float_as_uint(p);
            ph[n][i] = __builtin_bit_cast(__bf16, (uint16_t)(bits >> 16));
            pl[n][i] = (__bf16)(p - __uint_as_float(bits & 0xffff0000u));
          }
        const int key = kk * 32 + 4 * g + (ql >> 2);
#pragma unroll
        for (int d = 0; d < NDB; ++d) {
          const int j = d * 2 + ((ql >> 1) & 1);
          const char* v0 = vs + key * ROWB + ((j ^ vswz(key)) << 4) + (ql & 1) * 8;
          const char* v1 = vs + (key + 16) * ROWB + ((j ^ vswz(key + 16)) << 4) + (ql & 1) * 8;
          const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)v0);
          const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)v1);
          const auto w8 = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, w8);
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph[n], o[n][d], 0, 0, 0);
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[n], o[n][d], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = kb * 16 + 4 * g + i;
#pragma unroll
          for (int d = 0; d < NDB; ++d) {
            const int dim = d * 16 + ql;
            const float vf = *reinterpret_cast<const float*>(vs + key * ROWB + (((dim >> 2) ^ vswz(key)) << 4) + (dim & 3) * 4);
#pragma unroll
            for (int n = 0; n < NB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, sc[n][kb][i], o[n][d], 0, 0, 0);
          }
        }
    }
  }

  // Chunk w of V without its values that are not finite; true if there were any.  0
  // times such a value is not 0, so in tiles that not every query sees whole they are
  // left out of the product.
  static __device__ __forceinline__ bool finite(u32x4_t& w) {
    // an exponent of all ones overflows into the sign's place when one is added to it
    constexpr uint32_t EXP = BF ? 0x7f807f80u : 0x7f800000u, ONE = BF ? 0x00800080u : 0x00800000u;
    uint32_t over = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) over |= (w[e] & EXP) + ONE;
    const bool bad = (over & ~(EXP | (BF ? 0x007f007fu : 0x007fffffu))) != 0;
    if (bad) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF) {
          if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0x0000ffffu;
          if ((w[e] & 0x00007f80u) == 0x00007f80u) w[e] &= 0xffff0000u;
        } else {
          if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] = 0u;
        }
      }
    }
    return bad;
  }
  // ... and here they reach the rows that see them: p is positive there, so they are
  // what they add.  Dims (d0 + i * dstep) * 16 + 4g .. + 3 of query block n, from
  // the keys of `holes` alone, which has all that were left out.
  template <int ND>
  __device__ __forceinline__ void add_not_finite(const TreeAttnArgs& a, const Share& s, const Holes& holes, int n, int d0,
                                                 int dstep, f32x4_t (&x)[ND]) const {
    const int end = min(holes.end, s.kend);
    for (int key = holes.begin; key < end; ++key) {
      const int page = s.table[key >> a.shift];
      if ((unsigned)page >= (unsigned)a.n_pool) continue;
      const int j0 = key - s.ctx;
      uint64_t bits;
      if (a.mask) {
        MaskWords w;
        w.load(a.mask + qrow[n] * a.words, a.words, j0);
        bits = w.bits(j0);
      } else {
        bits = chain_bits(qi[n], j0);
      }
      if (!(bits & 1)) continue;
      const uint32_t row = page * a.v_page + (key & a.tail) * a.v_token;
      const T* vp = reinterpret_cast<const T*>(a.v + (uint64_t)row * a.unit + s.kvh * a.v_head);
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const int d = d0 + i * dstep;
        if (d >= NDB) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = St<T>::ld(vp + d * 16 + g * 4 + e);
          if (!(fabsf(v) < INFINITY)) x[i][e] += v;
        }
      }
    }
  }

  __device__ __forceinline__ void sum_lanes() {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      lsum[n] += __shfl_xor(lsum[n], 16);
      lsum[n] += __shfl_xor(lsum[n], 32);
    }
  }
  // Dims d * 16 + 4g .. + 3 of query block n: the result, or this split's part of it.
  __device__ __forceinline__ void put(const TreeAttnArgs& a, const Share& s, int n, int d, f32x4_t x, float mm,
                                      float ll) const {
    if (!qok[n]) return;
    const int64_t at = qrow[n] * a.H + qhead[n];
    if (s.nsplit > 1) {
      const int c = qi[n] * a.G + qhead[n] - s.kvh * a.G - s.q0;
      const int64_t pt = ((int64_t)s.unit * a.KH + s.kvh) * a.qb + c;
      *reinterpret_cast<f32x4_t*>(a.part + pt * DH + d * 16 + g * 4) = x;
      if (d == 0 && g == 0) a.part_ml[pt] = float2{mm, ll};
      return;
    }
    const bool some = ll > 0.f || ll != ll;
    x *= some ? 1.f / ll : 0.f;
    char* p = a.out + qrow[n] * a.o_row + qhead[n] * a.o_head + (d * 16 + g * 4) * (int)sizeof(T);
    if constexpr (BF) {
      bf16x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (__bf16)x[e];
      *reinterpret_cast<bf16x4_t*>(p) = w;
    } else {
      *reinterpret_cast<f32x4_t*>(p) = x;
    }
    if (a.lse && d == 0 && g == 0) a.lse[at] = some ? (mm + __log2f(ll)) * kLn2 : -INFINITY;
  }
};

// ---------------------------------------------------------------- few queries
// Up to 16 NQ queries a workgroup, all of them in each of its four waves; the waves take
// key tiles of their own in turn, staged through registers into a part of LDS that only
// they use, so there is no barrier until the four results are joined.  Bound by the reads
// of the cache: two workgroups of a CU hold 128 KB of rows in flight.
template <class T, int DH, int NQ, bool CUT>
__global__ void __launch_bounds__(256, 2) tree_attn_stream_kernel(TreeAttnArgs a) {
  constexpr int KW = sizeof(T) == 2 ? 32 : 16;
  typedef Tile<T, DH, NQ, KW> Tl;
  constexpr int CPR = Tl::CPR, ROWB = Tl::ROWB, NDB = Tl::NDB, NCH = KW * CPR / 64;
  __shared__ __align__(16) char lds[4 * 2 * Tl::BYTES];
  __shared__ float2 ml_s[4][16];
  __shared__ int2 holes_s[4];
  static_assert(4 * NDB * 64 * 16 <= 4 * 2 * Tl::BYTES, "the join fits the tiles");
  Share s;
  if (!s.init<CUT>(a)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* ks = lds + wave * 2 * Tl::BYTES;
  char* vs = ks + Tl::BYTES;
  const int first = s.kbeg + wave * KW;
  int pg = s.page(a, first, KW);
  TileRows rows;
  u32x4_t kreg[NCH], vreg[NCH];
  auto fetch = [&]() {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int key = (c * 64 + lane) / CPR, j = (c * 64 + lane) % CPR;
      kreg[c] = *reinterpret_cast<const u32x4_t*>(a.k + s.kvh * a.k_head + j * 16 + (uint64_t)__shfl(rows.k, key) * a.unit);
      vreg[c] = *reinterpret_cast<const u32x4_t*>(a.v + s.kvh * a.v_head + j * 16 + (uint64_t)__shfl(rows.v, key) * a.unit);
    }
  };
  rows.set(a, first, pg, Tl::ALL);
  if (first < s.kend) fetch();
  pg = s.page(a, first + 4 * KW, KW);
  Tl t;
  t.init(a, s, s.q0);
  const int i_first = s.q0 / a.G;
  Holes holes;

  for (int k0 = first; k0 < s.kend; k0 += 4 * KW) {
    const uint64_t there = rows.there;
    if (there != Tl::ALL || k0 + KW > s.clear) {
      bool bad = false;
#pragma unroll
      for (int c = 0; c < NCH; ++c) bad |= Tl::finite(vreg[c]);
      holes.add(there != 0 && __any(bad), k0, KW);
    }
    wave_sync();   // the lanes have read the tile before
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int key = (c * 64 + lane) / CPR, j = (c * 64 + lane) % CPR;
      *reinterpret_cast<u32x4_t*>(ks + key * ROWB + (j ^ Tl::kswz(key)) * 16) = kreg[c];
      *reinterpret_cast<u32x4_t*>(vs + key * ROWB + (j ^ Tl::vswz(key)) * 16) = vreg[c];
    }
    wave_sync();   // the tile is written
    if (k0 + 4 * KW < s.kend) {
      rows.set(a, k0 + 4 * KW, pg, Tl::ALL);
      fetch();
      pg = s.page(a, k0 + 8 * KW, KW);
    }
    const int j0 = k0 - s.ctx;
    const bool full = there == Tl::ALL && (j0 + KW <= 0 || (!a.mask && j0 + KW <= i_first + 1));
    uint64_t bits[NQ];
    if (!full) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if (a.mask) {
          MaskWords w;
          w.load(a.mask + t.qrow[n] * a.words, a.words, j0);
          bits[n] = there & w.bits(j0);
        } else {
          bits[n] = there & chain_bits(t.qi[n], j0);
        }
      }
    }
    t.template step<NQ>(a, ks, vs, full, bits, [](int) {});
  }

  const bool missing = holes.join(holes_s, wave);
  t.sum_lanes();
  // join of the four waves, 16 queries at a time; each wave writes a share of the dims, to
  // which it adds what was left out of them: behind the join, since the weight of a wave
  // that saw no key of a query is 0
  f32x4_t* ob = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    __syncthreads();
#pragma unroll
    for (int d = 0; d < NDB; ++d) ob[(wave * NDB + d) * 64 + lane] = t.o[n][d];
    if (t.g == 0) ml_s[wave][t.ql] = float2{t.m[n], t.lsum[n]};
    __syncthreads();
    float mm = -INFINITY, ll = 0.f, w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) mm = fmaxf(mm, ml_s[k][t.ql].x);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 x = ml_s[k][t.ql];
      w[k] = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - mm);
      ll += x.y * w[k];
    }
    constexpr int ND = (NDB + 3) / 4;
    f32x4_t x[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      x[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const int d = wave + i * 4;
      if (d < NDB)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[i] += ob[(k * NDB + d) * 64 + lane] * w[k];
    }
    if (missing) t.add_not_finite(a, s, holes, n, wave, 4, x);
#pragma unroll
    for (int i = 0; i < ND; ++i)
      if (wave + i * 4 < NDB) t.put(a, s, n, wave + i * 4, x[i], mm, ll);
  }
}

// ---------------------------------------------------------------- many queries
// 64 NQ queries a workgroup, 16 NQ in each of its four waves, all on the same key tiles.
// Tiles go from the cache to LDS without passing registers (global_load_lds, 1 KB a wave
// instruction: the swizzle is in which chunk a lane asks for), two stages, the next tile
// in flight during the present one's matrix work.  The loads are written so that the
// compiler does not count them; the wait for them is explicit.
template <class T, int DH, int NQ, bool CUT>
__global__ void __launch_bounds__(256, 2) tree_attn_tile_kernel(TreeAttnArgs a) {
  constexpr int KW = NQ * 8192 / (DH * (int)sizeof(T)) > 64 ? 64 : NQ * 8192 / (DH * (int)sizeof(T));
  typedef Tile<T, DH, NQ, KW> Tl;
  constexpr int CPR = Tl::CPR, NIN = Tl::BYTES / 4096;   // wave instructions per wave for K, and for V
  constexpr int KPI = 64 / CPR > 0 ? 64 / CPR : 1;        // keys of an instruction
  __shared__ __align__(1024) char lds[2 * 2 * Tl::BYTES];
  __shared__ int2 holes_s[4];
  Share s;
  if (!s.init<CUT>(a)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // A tile of up to 64 queries, a request's last: one block a wave instead of two for the
  // first waves (300 nodes x 128 users 1.24 -> 1.22 ms).
  const bool half = NQ == 2 && s.nq - s.q0 <= 64;
  const int first = s.q0 + wave * (half ? 16 : 16 * NQ);
  const bool active = first < s.nq;
  int pg = s.page(a, s.kbeg, KW);
  TileRows rows;
  // Wave instruction c of a tile's K (c < NIN) or V.  No memory clobber: what reads these
  // bytes stands behind the loop's wait and barrier, and the compiler is free to move the
  // present tile's reads past this.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int key0 = wave * KPI + lane / CPR;   // key of the lane in instruction 0; the next one's is 4 KPI on
  auto dma = [&](int c, int stage) {
    const bool v = c >= NIN;
    const int in = v ? c - NIN : c, key = key0 + in * 4 * KPI, j = lane % CPR;
    const uint32_t row = __builtin_amdgcn_ds_bpermute(key0 * 4 + in * 16 * KPI, v ? rows.v : rows.k);
    const char* p = (v ? a.v + s.kvh * a.v_head : a.k + s.kvh * a.k_head) +
                    (j ^ (v ? Tl::vswz(key) : Tl::kswz(key))) * 16 + (uint64_t)row * a.unit;
    const uint32_t at = lds0 + (stage * 2 + (v ? 1 : 0)) * Tl::BYTES + (in * 4 + wave) * 1024;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 ::"s"(__builtin_amdgcn_readfirstlane(at)), "v"(p) : "m0");
  };
  // A CU takes one such instruction in 16 clocks: issued all at once behind the barrier,
  // they hold up the four waves for 500, so they go between the matrix instructions.
  constexpr int PER = (2 * NIN + Tl::NKS - 1) / Tl::NKS;
  auto some_dma = [&](int k, int stage) {
#pragma unroll
    for (int c = k * PER; c < (k + 1) * PER; ++c)
      if (c < 2 * NIN) dma(c, stage);
  };
  auto fetch = [&](int stage) {
#pragma unroll
    for (int k = 0; k < Tl::NKS; ++k) some_dma(k, stage);
  };
  rows.set(a, s.kbeg, pg, Tl::ALL);
  if (s.kbeg < s.kend) fetch(0);
  pg = s.page(a, s.kbeg + KW, KW);
  Tl t;
  t.init(a, s, active ? first : s.nq - 1);
  const int i_first = (active ? first : s.nq - 1) / a.G;
  Holes holes;
  auto run = [&](auto blocks) {
    constexpr int NB = decltype(blocks)::value;
    MaskWords words[NB];
    auto load_words = [&](int k0) {
      if (a.mask && k0 + KW > s.ctx) {
#pragma unroll
        for (int n = 0; n < NB; ++n) words[n].load(a.mask + t.qrow[n] * a.words, a.words, k0 - s.ctx);
      }
    };
    load_words(s.kbeg);

    int stage = 0;
    for (int k0 = s.kbeg; k0 < s.kend; k0 += KW, stage ^= 1) {
      const uint64_t there = rows.there;
      char* ks = lds + stage * 2 * Tl::BYTES;
      char* vs = ks + Tl::BYTES;
      const int j0 = k0 - s.ctx;
      const bool full = there == Tl::ALL && (j0 + KW <= 0 || (!a.mask && j0 + KW <= i_first + 1));
      uint64_t bits[NQ];
      if (!full) {
#pragma unroll
        for (int n = 0; n < NB; ++n) bits[n] = there & (a.mask ? words[n].bits(j0) : chain_bits(t.qi[n], j0));
      }
      // this tile has landed, and the other stage has been read
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      const bool more = k0 + KW < s.kend;
      if (more) {
        rows.set(a, k0 + KW, pg, Tl::ALL);
        load_words(k0 + KW);
        pg = s.page(a, k0 + 2 * KW, KW);
      }
      if (there != Tl::ALL || k0 + KW > s.clear) {
        bool bad = false;
#pragma unroll
        for (int c = 0; c < NIN; ++c) {
          u32x4_t* p = reinterpret_cast<u32x4_t*>(vs) + c * 256 + threadIdx.x;
          u32x4_t w = *p;
          if (Tl::finite(w)) {
            *p = w;
            bad = true;
          }
        }
        holes.add(there != 0 && __any(bad), k0, KW);
        __syncthreads();
      }
      bool some = full;
      if (!full) {
        uint64_t any = 0;
#pragma unroll
        for (int n = 0; n < NB; ++n) any |= bits[n];
        some = __any(any != 0);
      }
      if (!active || !some) {   // no query of the wave sees the tile
        if (more) fetch(stage ^ 1);
      } else {
        // the last tile asks for itself again: without a branch here the matrix
        // instructions stay in one block (causal chunks 117 us with it, 107 without)
        t.template step<NB>(a, ks, vs, full, bits, [&](int k) { some_dma(k, stage ^ 1); });
      }
    }
  };
  if (half) run(std::integral_constant<int, 1>{});
  else run(std::integral_constant<int, NQ>{});
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is written to LDS behind the workgroup's end
  const bool missing = holes.join(holes_s, wave);
  t.sum_lanes();
  if (!active) return;
  if (missing) {
#pragma unroll
    for (int n = 0; n < NQ; ++n)
      if (n == 0 || !half) t.add_not_finite(a, s, holes, n, 0, 1, t.o[n]);
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n)
    if (n == 0 || !half)
#pragma unroll
      for (int d = 0; d < Tl::NDB; ++d) t.put(a, s, n, d, t.o[n][d], t.m[n], t.lsum[n]);
}

// Joins the parts of requests whose keys were split.  DH / 4 threads, a group, hold a
// row and head, four dims each.  Bound by the latency of the loads, so many parts (MANY)
// get a workgroup per row and head: all threads take the parts' maxima and sums, then its
// groups the parts in turn (61 parts of 4 users' 32 rows: 29 us with a group for each
// row, 14 so).  Few parts get a group.
template <class T, int DH, bool MANY>
__global__ void __launch_bounds__(256) tree_attn_join_kernel(TreeAttnArgs a) {
  constexpr int LPR = DH / 4, GROUPS = 256 / LPR;
  const int tid = threadIdx.x, lane = tid % LPR, grp = tid / LPR;
  const int at = MANY ? blockIdx.x : blockIdx.x * GROUPS + grp;
  const int h = at % a.H, bi = at / a.H, b = bi / a.max_new, i = bi % a.max_new;
  if (b >= a.B) return;
  int r0;
  const int count = new_rows(a, b, r0);
  if (i >= min(count, a.n_rows - r0)) return;
  const int4 where = a.split[b];   // first unit, parts, tiles
  const int n = where.y, q = i * a.G + h % a.G;
  if (n <= 1) return;
  const int64_t out_row = (int64_t)r0 + i, row = ((int64_t)(where.x + q / a.qb) * a.KH + h / a.G) * a.qb + q % a.qb,
                step = (int64_t)where.z * a.KH * a.qb;
  const f32x4_t* part = reinterpret_cast<const f32x4_t*>(a.part + row * DH) + lane;
  float mm = -INFINITY, ll = 0.f;
  auto weight = [&](float m) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm); };
  f32x4_t x = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if constexpr (MANY) {
    __shared__ f32x4_t xs[GROUPS][LPR];
    __shared__ float red[2][4];
    for (int k = tid; k < n; k += 256) mm = fmaxf(mm, a.part_ml[k * step + row].x);
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) mm = fmaxf(mm, __shfl_xor(mm, w));
    if ((tid & 63) == 0) red[0][tid >> 6] = mm;
    __syncthreads();
    mm = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    for (int k = tid; k < n; k += 256) {
      const float2 ml = a.part_ml[k * step + row];
      ll += ml.y * weight(ml.x);
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) ll += __shfl_xor(ll, w);
    if ((tid & 63) == 0) red[1][tid >> 6] = ll;
#pragma unroll 4
    for (int k = grp; k < n; k += GROUPS) x += part[k * step * LPR] * weight(a.part_ml[k * step + row].x);
    xs[grp][lane] = x;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) x += xs[k][lane];
    ll = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  } else {
#pragma unroll 4
    for (int k = 0; k < n; ++k) mm = fmaxf(mm, a.part_ml[k * step + row].x);
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
      const float2 ml = a.part_ml[k * step + row];
      const float w = weight(ml.x);
      x += part[k * step * LPR] * w;
      ll += ml.y * w;
    }
  }
  const bool some = ll > 0.f || ll != ll;
  x *= some ? 1.f / ll : 0.f;
  T* out = reinterpret_cast<T*>(a.out + out_row * a.o_row + h * a.o_head) + lane * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) St<T>::st(out + e, x[e]);
  if (a.lse && lane == 0) a.lse[out_row * a.H + h] = some ? (mm + __log2f(ll)) * kLn2 : -INFINITY;
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
  if (a.n_rows >= (1 << 30)) return fail(ATSPEED_E_SHAPE, "n_rows must be below 2^30");
  if ((long long)a.n_rows * a.n_heads >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "n_rows x n_heads must be below 2^31");
  return ATSPEED_OK;
}

}  // namespace atspeed

using namespace atspeed;

namespace {

// Launch of one call: queries per workgroup, and how the keys are split.
struct AttnPlan {
  int tile;          // queries of a workgroup
  int qtiles, units, cap;
  size_t part_at, ml_at, bytes;   // of the workspace
};

AttnPlan plan_attention(const atspeed_tree_attention_args& a) {
  AttnPlan p{};
  const bool bf = a.dtype == ATSPEED_BF16;
  const int64_t nq = (int64_t)std::min(a.max_new, a.n_rows) * (a.n_heads / a.n_kv_heads);
  const int64_t pairs = (int64_t)a.B * a.n_kv_heads;
  p.cap = (int)std::min<int64_t>((int64_t)a.max_pages * a.page_size, 1 << 30);
  const int64_t keys = std::max<int64_t>(1, std::min<int64_t>((int64_t)a.max_ctx + a.max_new, p.cap));
  // Queries of a workgroup: the smallest tile that holds them.  fp32 has tiles of 16, 32
  // and 64; those of 32 take the registers of d_head 128 and, with d_head 64, half of the
  // waves of a CU, which pays below 256 workgroups (fp32 in tiles of 64 and of 32, us: 24
  // rows x 40 users over 300 keys, 12 heads of 32, 15.7 and 10.4; 4 rows x 2 users over
  // 6,000 keys, 32 heads of 64 on 4, 21.8 and 16.6; but 18 rows x 30 users over 150 keys, 32
  // heads of 64, 15.6 and 19.1).
  // Launches that do not fill the CUs are bound by the steps each workgroup takes one
  // after the other; over up to 1,024 keys they take the tiles of few queries, whose four
  // waves share the steps out, though these read the keys once for each: up to 256 of
  // them, and up to 1,024 where the larger tiles are 256 at most (fp32, whose matrix
  // instructions are slower, 384) and the keys more than a step (us, larger tiles and
  // few: 30 rows over 110 keys, fp32, d_head 32, 7.2 and 5.0; 100 rows x 20 users over 600
  // keys, 8 heads of 64, 17.0 and 9.3; 900 rows x 4 users over 1,000, 23.8 and 12.0; 50
  // rows x 30 users over 300 keys, fp32, 20.4 and 16.1; but 12 rows x 50 users over 600
  // keys, 32 heads on 8, 400 larger tiles, 21.9 and 25.7; 60 rows x 56 users over 502
  // keys, fp32, 448 larger ones, 25.9 and 30.5; 50 rows x 32 users over 80 keys 8.0 and 9.9).
  const int few = bf || (a.d_head <= 64 && pairs * ((nq + 15) / 16) > 256) ? 32 : 16, few_step = bf ? 128 : 64;
  p.tile = nq <= 16 ? 16 : nq <= 32 && (bf || a.d_head == 32 || (a.d_head == 64 && pairs <= 256)) ? 32 : nq <= 64 || !bf ? 64 : 128;
  const int64_t in_few = pairs * ((nq + few - 1) / few), in_tiles = pairs * ((nq + p.tile - 1) / p.tile);
  if (p.tile > few && keys <= 1024 &&
      (in_few <= 256 || (keys > few_step && in_few <= 1024 && in_tiles <= (bf ? 256 : 384))))
    p.tile = few;
  p.qtiles = (int)((nq + p.tile - 1) / p.tile);
  // Requests are split where the launch has at least two pieces a tile of queries: into
  // 512 workgroups, two for each of the 256 CUs, or as few times that as it takes, all of
  // the same length as far as the contexts allow, since the kernel has them (Share::pick).
  // Pieces of one length as the host alone could cut them, for the longest context, took
  // (us; so): trees of 4 users over up to 65,536 keys 144 (136); of one over 65,536 102
  // (71); one prompt chunk of 1,024 rows over 4,096 keys 137 (114), 300 rows over 30,000,
  // 2 heads, 211 (80); 64 single tokens over up to 8,192 keys 148 (145).  1,024 workgroups
  // for the second and third take 90 and 130: each piece pays its start and its part.
  // Pieces of under 256 keys lose to their join, and so does any split of up to 10 steps
  // (4 rows x 8 users over 600 keys: 10.2 us in pieces, 8.3 whole; 256 rows x 8 users over
  // 310 keys 31 and 14).
  const int step = p.tile <= 32 ? few_step : std::min(64, (p.tile / 64) * 8192 / (a.d_head * (bf ? 2 : 4)));
  const int64_t tiles = (int64_t)a.B * p.qtiles;
  int64_t units = std::max(1, 512 / a.n_kv_heads);
  while (units < 2 * tiles && units * 2 * a.n_kv_heads <= 2048) units *= 2;
  if (keys > 10 * step && units >= 2 * tiles) {
    p.units = (int)units;
    const size_t rows = (size_t)units * a.n_kv_heads * p.tile;
    p.part_at = (size_t)a.B * sizeof(int4);
    p.ml_at = p.part_at + rows * a.d_head * sizeof(float);
    p.bytes = p.ml_at + rows * sizeof(float2);
  }
  return p;
}

template <class T, int DH, class F>
atspeed_status launch_attention(const TreeAttnArgs& p, F kernel, hipStream_t st) {
  const long long pairs = (long long)p.B * p.KH;
  const long long n = p.units ? (p.units * p.KH + 7) / 8 * 8 : (pairs + 7) / 8 * 8 * p.qtiles;
  if (n > kMaxGroups) return fail(ATSPEED_E_SHAPE, "tree attention: too many query tiles");
  hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(256), 0, st, p);
  HIP_TRY(hipGetLastError());
  if (p.units) {
    // few: units come only with few query tiles
    const unsigned rows = (unsigned)((long long)p.B * p.max_new * p.H), groups = 1024 / DH;
    if (p.units <= 16 * p.B * p.qtiles)
      hipLaunchKernelGGL((tree_attn_join_kernel<T, DH, false>), dim3((rows + groups - 1) / groups), dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL((tree_attn_join_kernel<T, DH, true>), dim3(rows), dim3(256), 0, st, p);
    HIP_TRY(hipGetLastError());
  }
  return ATSPEED_OK;
}

template <class T, int DH, bool CUT>
atspeed_status run_attention(const TreeAttnArgs& p, hipStream_t st) {
  if (p.qb == 16) return launch_attention<T, DH>(p, tree_attn_stream_kernel<T, DH, 1, CUT>, st);
  if (p.qb == 64) return launch_attention<T, DH>(p, tree_attn_tile_kernel<T, DH, 1, CUT>, st);
  if constexpr (sizeof(T) == 2 || DH <= 64) {
    if (p.qb == 32) return launch_attention<T, DH>(p, tree_attn_stream_kernel<T, DH, 2, CUT>, st);
  }
  if constexpr (sizeof(T) == 2) {
    return launch_attention<T, DH>(p, tree_attn_tile_kernel<T, DH, 2, CUT>, st);
  }
  return fail(ATSPEED_E_DEVICE, "tree attention: no such tile");
}

template <class T, int DH>
atspeed_status run_attention(const TreeAttnArgs& p, hipStream_t st) {
  return p.units ? run_attention<T, DH, true>(p, st) : run_attention<T, DH, false>(p, st);
}

}  // namespace

extern "C" {

atspeed_status atspeed_tree_attention_workspace_bytes(const atspeed_tree_attention_args* args, size_t* bytes) {
  if (!bytes) return fail(ATSPEED_E_INVALID, "bytes is null");
  ST_TRY(check_attention(args));
  *bytes = plan_attention(*args).bytes;
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
  const AttnPlan plan = plan_attention(a);
  if (plan.bytes && (!workspace || !aligned16(workspace) || ws_bytes < plan.bytes))
    return fail(ATSPEED_E_WORKSPACE, "tree attention: workspace is too small or not 16-byte aligned");
  TreeAttnArgs p{};
  p.q = (const char*)a.q; p.q_row = a.q_row_stride * es; p.q_head = a.q_head_stride * es;
  p.k = (const char*)a.k_pages.data; p.v = (const char*)a.v_pages.data;
  p.k_head = a.k_pages.head_stride * es; p.v_head = a.v_pages.head_stride * es;
  // rows of the caches by 32-bit numbers of the largest unit that divides the strides
  const int64_t strides[] = {a.k_pages.page_stride * es, a.k_pages.token_stride * es, a.v_pages.page_stride * es,
                             a.v_pages.token_stride * es};
  uint64_t any = 1u << 20;
  for (int64_t s : strides) {
    if (s < 0) return fail(ATSPEED_E_INVALID, "tree attention: negative cache strides");
    any |= (uint64_t)s;
  }
  p.unit = (uint32_t)(any & (~any + 1));
  for (int i = 0; i < 4; i += 2)
    if ((double)strides[i] / p.unit * a.n_pool + (double)strides[i + 1] / p.unit * a.page_size >= 4294967296.0)
      return fail(ATSPEED_E_SHAPE, "tree attention: a cache of 2^32 or more of the largest unit dividing its strides");
  p.k_page = (uint32_t)(strides[0] / p.unit); p.k_token = (uint32_t)(strides[1] / p.unit);
  p.v_page = (uint32_t)(strides[2] / p.unit); p.v_token = (uint32_t)(strides[3] / p.unit);
  p.table = a.block_table; p.row_off = a.row_off; p.ctx = a.ctx; p.mask = a.mask;
  p.out = (char*)a.out; p.o_row = a.out_row_stride * es; p.o_head = a.out_head_stride * es;
  p.lse = a.lse;
  p.split = (int4*)workspace;
  p.part = (float*)((char*)workspace + plan.part_at); p.part_ml = (float2*)((char*)workspace + plan.ml_at);
  p.B = a.B; p.n_rows = a.n_rows; p.H = a.n_heads; p.KH = a.n_kv_heads; p.G = a.n_heads / a.n_kv_heads;
  p.max_pages = a.max_pages; p.n_pool = a.n_pool; p.max_new = std::min(a.max_new, a.n_rows); p.words = a.mask_words;
  p.shift = log2_of(a.page_size); p.tail = a.page_size - 1;
  p.qtiles = plan.qtiles; p.qb = plan.tile; p.units = plan.units; p.cap = plan.cap;
  // the queries carry the scale's sign, so that the largest product is the largest score
  p.q_flip = a.scale < 0.f ? (es == 2 ? 0x80008000u : 0x80000000u) : 0u;
  p.scale = std::max(std::fabs(a.scale) * 1.4426950408889634f, 1e-37f);
  hipStream_t st = (hipStream_t)stream;
  if (es == 2) return a.d_head == 64 ? run_attention<bf16_t, 64>(p, st) : run_attention<bf16_t, 128>(p, st);
  if (a.d_head == 32) return run_attention<float, 32>(p, st);
  if (a.d_head == 64) return run_attention<float, 64>(p, st);
  return run_attention<float, 128>(p, st);
}

}  // extern "C"
