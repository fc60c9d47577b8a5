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
  float* part;                 // [splits][n_rows][H][d_head] unnormalised sums of split requests
  float2* part_ml;             // [splits][n_rows][H] running maximum and sum
  int B, n_rows, H, G, KH, max_pages, n_pool, max_new, words, shift, tail;
  int qtiles, splits;
  int64_t chunk;               // keys of a split
  uint32_t q_flip;             // sign bits of the queries' elements (negative scale)
  float scale;                 // |scale| log2(e)
};

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // a maximum moves when a score passes it by 2^8

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// Keys of a request as the rows of one query tile see them.
struct KeySpan {
  int64_t ctx;      // context keys (0 where the request sees nothing)
  int64_t total;    // keys of the request: what the splits divide
};
__device__ __forceinline__ KeySpan key_span(const TreeAttnArgs& a, int b, int count) {
  const int64_t ctx = a.ctx[b];
  if (ctx < 0) return {0, 0};
  const int64_t cap = (int64_t)a.max_pages << a.shift;
  return {ctx < cap ? ctx : cap, min(ctx + (a.mask ? min((int64_t)count, (int64_t)a.words * 64) : (int64_t)count), cap)};
}

// Bits kk of a 64-key tile at k0 that the row sees: context keys, then its mask words
// (or the keys up to its own, at ctx + i).
__device__ __forceinline__ uint64_t tile_bits(const uint64_t* words, int n_words, int64_t ctx, int i, int64_t k0) {
  const int64_t j0 = k0 - ctx;
  if (!words) {
    const int64_t n = i + 1 - j0;
    return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
  }
  if (j0 <= -64) return ~0ull;
  if (j0 < 0) return (words[0] << -j0) | ((1ull << -j0) - 1);
  const int64_t w = j0 >> 6;
  const int sh = (int)(j0 & 63);
  const uint64_t lo = w < n_words ? words[w] >> sh : 0ull;
  const uint64_t hi = sh && w + 1 < n_words ? words[w + 1] << (64 - sh) : 0ull;
  return lo | hi;
}

// Pieces of a request's keys; the last one takes what a context above max_ctx holds more.
__device__ __forceinline__ int split_count(const TreeAttnArgs& a, int64_t total) {
  return total <= a.chunk ? 1 : (int)min((total + a.chunk - 1) / a.chunk, (int64_t)a.splits);
}

template <class T, int DH, int NQ, int WQ, int KW>
__global__ void __launch_bounds__(256)
tree_attn_kernel(TreeAttnArgs a) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int WK = 4 / WQ;                    // key groups
  constexpr int TG = 64 * WQ;                   // threads of a key group
  constexpr int ROWB = DH * (int)sizeof(T);     // bytes of a row
  constexpr int CPR = ROWB / 16;                // 16-byte chunks of a row
  constexpr int NKS = CPR / 4;                  // chunk groups of a score
  constexpr int NDB = DH / 16;                  // 16-dim blocks of the output
  constexpr int NKB = KW / 16;                  // 16-key blocks of a tile
  constexpr int NCH = KW * CPR / TG;            // chunks of K (and of V) a thread stages
  constexpr int QB = 16 * NQ * WQ;              // queries of a workgroup
  constexpr int TILE = KW * ROWB;
  constexpr int JOIN = WK > 1 ? 4 * NDB * 64 * 16 : 0;
  constexpr int LDS = WK * 2 * TILE > JOIN ? WK * 2 * TILE : JOIN;
  __shared__ __align__(16) char lds[LDS];
  __shared__ float2 ml_s[4][16];
  auto kswz = [](int key) { return BF ? key & (CPR - 1) : CPR >= 16 ? key & 15 : (key >> 1) & 7; };
  auto vswz = [](int key) {
    return BF ? (DH == 128 ? key & 7 : (key >> 1) & 3) << 1 : ((key >> 2) & (NDB >= 4 ? 3 : 1)) << 2;
  };

  const int Lw = blockIdx.x, xcd = Lw & 7, rest = Lw >> 3, Z = a.qtiles * a.splits;
  const int pair = (rest / Z) * 8 + xcd, z = rest % Z;
  if (pair >= a.B * a.KH) return;
  const int b = pair / a.KH, kvh = pair % a.KH;
  const int split = z / a.qtiles, qt = a.mask ? z % a.qtiles : a.qtiles - 1 - z % a.qtiles;   // chains: longest first
  const int r0 = a.row_off[b], count = a.row_off[b + 1] - r0;
  const int nr = min(min(count, a.n_rows - r0), a.max_new);
  const int nq = nr * a.G, q0 = qt * QB;
  if (q0 >= nq) return;
  const KeySpan span = key_span(a, b, count);
  const int nsplit = split_count(a, span.total);
  if (split >= nsplit) return;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wq = wave % WQ, wk = wave / WQ, gt = wq * 64 + lane;
  const int g = lane >> 4, ql = lane & 15;
  char* ks = lds + wk * 2 * TILE;
  char* vs = ks + TILE;

  // this lane's queries, one per 16-query block
  int qi[NQ];           // new-row index
  int64_t qrow[NQ];
  int qhead[NQ];
  bool qok[NQ];
  f32x4_t qf[NQ][NKS];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int c = q0 + (wq * NQ + n) * 16 + ql;
    qok[n] = c < nq;
    const int cc = qok[n] ? c : nq - 1;
    qi[n] = cc / a.G;
    qrow[n] = r0 + qi[n];
    qhead[n] = kvh * a.G + cc % a.G;
    const char* p = a.q + qrow[n] * a.q_row + qhead[n] * a.q_head + g * 16;
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      u32x4_t w = *reinterpret_cast<const u32x4_t*>(p + s * 64);
      w ^= a.q_flip;
      qf[n][s] = __builtin_bit_cast(f32x4_t, w);
    }
  }
  const int i_first = (q0 + wq * NQ * 16 < nq ? q0 + wq * NQ * 16 : nq - 1) / a.G;   // first row of the wave
  const int i_last = (min(q0 + QB, nq) - 1) / a.G;                                    // last row of the workgroup
  const int64_t kbeg = split * a.chunk;
  int64_t kend = split + 1 < nsplit ? kbeg + a.chunk : span.total;
  if (!a.mask) kend = min(kend, span.ctx + i_last + 1);
  // from this key on some query of the workgroup may not see a key
  const int64_t clear = a.mask ? span.ctx : span.ctx + q0 / a.G + 1;
  const int nit = kend > kbeg ? (int)((kend - kbeg + WK * KW - 1) / (WK * KW)) : 0;
  const int* table = a.table + (int64_t)b * a.max_pages;

  auto key0 = [&](int it) { return kbeg + (int64_t)(it * WK + wk) * KW; };
  // page of key k0 + lane, -1 where there is none
  auto load_page = [&](int it) {
    const int64_t key = key0(it) + lane;
    int pg = -1;
    if (lane < KW && key < kend) pg = table[key >> a.shift];
    return pg;
  };
  u32x4_t kreg[NCH], vreg[NCH];
  auto fetch = [&](int it, int pg) {
    const int64_t k0 = key0(it);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int idx = gt + c * TG, key = idx / CPR, j = idx % CPR;
      const int page = __shfl(pg, key);
      const int64_t tok = (k0 + key) & a.tail;
      kreg[c] = vreg[c] = u32x4_t{0u, 0u, 0u, 0u};
      if ((unsigned)page < (unsigned)a.n_pool) {
        kreg[c] = *reinterpret_cast<const u32x4_t*>(a.k.data + page * a.k.page + tok * a.k.token + kvh * a.k.head + j * 16);
        vreg[c] = *reinterpret_cast<const u32x4_t*>(a.v.data + page * a.v.page + tok * a.v.token + kvh * a.v.head + j * 16);
      }
    }
  };

  f32x4_t o[NQ][NDB];
  float m[NQ], lsum[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -INFINITY;
    lsum[n] = 0.f;
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[n][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  bool bad = false;                    // a value that not every query sees is not finite
  const uint64_t whole = KW == 64 ? ~0ull : (1ull << KW) - 1;
  int pg = load_page(0);
  uint64_t vm = __ballot((unsigned)pg < (unsigned)a.n_pool);
  if (nit > 0) fetch(0, pg);
  pg = load_page(1);

  for (int it = 0; it < nit; ++it) {
    const int64_t k0 = key0(it);
    const bool partial = k0 + KW > clear;
    if (partial) {
      // 0 times a value that is not finite is not 0: such values are left out of the
      // product and reach the rows that see them below
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = vreg[c][e];
          if constexpr (BF) {
            if ((w & 0x7f800000u) == 0x7f800000u) { vreg[c][e] &= 0x0000ffffu; bad = true; }
            if ((w & 0x00007f80u) == 0x00007f80u) { vreg[c][e] &= 0xffff0000u; bad = true; }
          } else {
            if ((w & 0x7f800000u) == 0x7f800000u) { vreg[c][e] = 0u; bad = true; }
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int idx = gt + c * TG, key = idx / CPR, j = idx % CPR;
      *reinterpret_cast<u32x4_t*>(ks + key * ROWB + (j ^ kswz(key)) * 16) = kreg[c];
      *reinterpret_cast<u32x4_t*>(vs + key * ROWB + (j ^ vswz(key)) * 16) = vreg[c];
    }
    if (WQ > 1) __syncthreads();
    const uint64_t tile_vm = vm;
    if (it + 1 < nit) {
      vm = __ballot((unsigned)pg < (unsigned)a.n_pool);
      fetch(it + 1, pg);
      pg = load_page(it + 2);
    }
    // scores
    f32x4_t sc[NQ][NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      const int key = kb * 16 + ql;
#pragma unroll
      for (int n = 0; n < NQ; ++n) sc[n][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NKS; ++s) {
        const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(ks + key * ROWB + ((s * 4 + g) ^ kswz(key)) * 16);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          if constexpr (BF) {
            sc[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf),
                                                                 __builtin_bit_cast(bf16x8_t, qf[n][s]), sc[n][kb], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[n][kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[n][s][e], sc[n][kb], 0, 0, 0);
          }
        }
      }
    }
    const bool full = tile_vm == whole && (k0 + KW <= span.ctx || (!a.mask && k0 + KW <= span.ctx + i_first + 1));
    float mx[NQ];
    bool moved = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      if (!full) {
        const uint64_t bits =
            tile_vm & tile_bits(a.mask ? a.mask + qrow[n] * a.words : nullptr, a.words, span.ctx, qi[n], k0);
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((bits >> (kb * 16 + g * 4 + i)) & 1)) sc[n][kb][i] = -INFINITY;
      }
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
      for (int n = 0; n < NQ; ++n) {
        float x = fmaxf(mx[n], __shfl_xor(mx[n], 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        const float mnew = fmaxf(m[n], x);
        const float alpha = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - mnew);
        m[n] = mnew;
        lsum[n] *= alpha;
#pragma unroll
        for (int d = 0; d < NDB; ++d) o[n][d] *= alpha;
      }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float ref = m[n] != -INFINITY ? m[n] : 0.f;
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
    // values
    if constexpr (BF) {
#pragma unroll
      for (int kk = 0; kk < KW / 32; ++kk) {
        bf16x8_t pf[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pf[n][i] = (__bf16)sc[n][2 * kk][i];
            pf[n][4 + i] = (__bf16)sc[n][2 * kk + 1][i];
          }
        const int key = kk * 32 + 4 * g + (ql >> 2);
#pragma unroll
        for (int d = 0; d < NDB; ++d) {
          const int j = d * 2 + ((ql >> 1) & 1);
          char* v0 = vs + key * ROWB + ((j ^ vswz(key)) << 4) + (ql & 1) * 8;
          char* v1 = vs + (key + 16) * ROWB + ((j ^ vswz(key + 16)) << 4) + (ql & 1) * 8;
          const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)v0);
          const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)v1);
          const auto w8 = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, w8);
#pragma unroll
          for (int n = 0; n < NQ; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[n][d], 0, 0, 0);
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
            for (int n = 0; n < NQ; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, sc[n][kb][i], o[n][d], 0, 0, 0);
          }
        }
    }
    if (WQ > 1) __syncthreads();
  }

  if (__syncthreads_or(bad) && wk == 0) {
    // p is positive where the row sees the key, so such a value is what it adds
    for (int64_t key = max(kbeg, clear - KW); key < kend; ++key) {
      const int page = table[key >> a.shift];
      if ((unsigned)page >= (unsigned)a.n_pool) continue;
      const char* vp = a.v.data + page * a.v.page + (key & a.tail) * a.v.token + kvh * a.v.head;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if (!(tile_bits(a.mask ? a.mask + qrow[n] * a.words : nullptr, a.words, span.ctx, qi[n], key) & 1)) continue;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = St<T>::ld(reinterpret_cast<const T*>(vp) + d * 16 + g * 4 + e);
            if (!(fabsf(v) < INFINITY)) o[n][d][e] += v;
          }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    lsum[n] += __shfl_xor(lsum[n], 16);
    lsum[n] += __shfl_xor(lsum[n], 32);
  }

  // dims d * 16 + 4 g .. + 3 of one query: the result, or this split's part of it
  auto put = [&](int n, int d, f32x4_t x, float mm, float ll) {
    if (!qok[n]) return;
    if (nsplit > 1) {
      const int64_t at = (split * (int64_t)a.n_rows + qrow[n]) * a.H + qhead[n];
      *reinterpret_cast<f32x4_t*>(a.part + at * DH + d * 16 + g * 4) = x;
      if (d == 0 && g == 0) a.part_ml[at] = float2{mm, ll};
      return;
    }
    const float inv = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
    x *= inv;
    char* p = a.out + qrow[n] * a.o_row + qhead[n] * a.o_head + (d * 16 + g * 4) * (int)sizeof(T);
    if constexpr (BF) {
      typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
      bf16x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (__bf16)x[e];
      *reinterpret_cast<bf16x4_t*>(p) = w;
    } else {
      *reinterpret_cast<f32x4_t*>(p) = x;
    }
    if (a.lse && d == 0 && g == 0)
      a.lse[qrow[n] * a.H + qhead[n]] = ll > 0.f || ll != ll ? (mm + __log2f(ll)) * kLn2 : -INFINITY;
  };
  if constexpr (WK == 1) {
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int d = 0; d < NDB; ++d) put(n, d, o[n][d], m[n], lsum[n]);
  } else {
    // join of the key groups: each block of 16 queries through LDS, the output's dims shared out
    f32x4_t* ob = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      __syncthreads();
#pragma unroll
      for (int d = 0; d < NDB; ++d) ob[(wave * NDB + d) * 64 + lane] = o[n][d];
      if (g == 0) ml_s[wave][ql] = float2{m[n], lsum[n]};
      __syncthreads();
      float mm = -INFINITY, ll = 0.f, w[WK];
#pragma unroll
      for (int k = 0; k < WK; ++k) mm = fmaxf(mm, ml_s[k * WQ + wq][ql].x);
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float2 x = ml_s[k * WQ + wq][ql];
        w[k] = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - mm);
        ll += x.y * w[k];
      }
      for (int d = wk; d < NDB; d += WK) {
        f32x4_t x = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WK; ++k) x += ob[((k * WQ + wq) * NDB + d) * 64 + lane] * w[k];
        put(n, d, x, mm, ll);
      }
    }
  }
}

// Joins the parts of requests whose keys were split: DH / 4 lanes per row and head.
template <class T, int DH>
__global__ void __launch_bounds__(256) tree_attn_join_kernel(TreeAttnArgs a) {
  constexpr int LPR = DH / 4;
  const int64_t idx = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const int lane = threadIdx.x % LPR, h = (int)(idx % a.H);
  const int64_t bi = idx / a.H;
  const int b = (int)(bi / a.max_new), i = (int)(bi % a.max_new);
  if (b >= a.B) return;
  const int r0 = a.row_off[b], count = a.row_off[b + 1] - r0;
  if (i >= min(count, a.n_rows - r0)) return;
  const KeySpan span = key_span(a, b, count);
  const int n = split_count(a, span.total);
  if (n <= 1) return;
  const int64_t row = ((int64_t)r0 + i) * a.H + h, step = (int64_t)a.n_rows * a.H;
  float mm = -INFINITY;
  for (int s = 0; s < n; ++s) mm = fmaxf(mm, a.part_ml[s * step + row].x);
  float ll = 0.f;
  f32x4_t x = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < n; ++s) {
    const float2 ml = a.part_ml[s * step + row];
    const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mm);
    ll += ml.y * w;
    x += *reinterpret_cast<const f32x4_t*>(a.part + (s * step + row) * DH + lane * 4) * w;
  }
  const bool some = ll > 0.f || ll != ll;
  x *= some ? 1.f / ll : 0.f;
  T* out = reinterpret_cast<T*>(a.out + ((int64_t)r0 + i) * a.o_row + h * a.o_head) + lane * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) St<T>::st(out + e, x[e]);
  if (a.lse && lane == 0) a.lse[row] = some ? (mm + __log2f(ll)) * kLn2 : -INFINITY;
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

namespace {

// Launch of one call: queries per workgroup, and how the keys are split.
struct AttnPlan {
  int tile;          // queries of a workgroup
  int qtiles, splits;
  int64_t chunk;
  size_t part_bytes, bytes;
};

AttnPlan plan_attention(const atspeed_tree_attention_args& a) {
  AttnPlan p{};
  const int64_t nq = (int64_t)std::min(a.max_new, a.n_rows) * (a.n_heads / a.n_kv_heads);
  p.tile = nq <= 16 ? 16 : nq <= 32 ? 32 : nq <= 64 ? 64 : 128;
  p.qtiles = (int)((nq + p.tile - 1) / p.tile);
  const int64_t cap = (int64_t)a.max_pages * a.page_size;
  const int64_t keys = std::max<int64_t>(1, std::min<int64_t>((int64_t)a.max_ctx + a.max_new, cap));
  const int64_t base = (int64_t)a.B * a.n_kv_heads * p.qtiles;
  const int64_t want = std::max<int64_t>(1, 2048 / base);
  p.chunk = std::max<int64_t>(256, ((keys + want - 1) / want + 127) / 128 * 128);
  p.splits = (int)((keys + p.chunk - 1) / p.chunk);
  const size_t rows = (size_t)p.splits * a.n_rows * a.n_heads;
  p.part_bytes = p.splits > 1 ? rows * a.d_head * sizeof(float) : 0;
  p.bytes = p.splits > 1 ? p.part_bytes + rows * sizeof(float2) : 0;
  return p;
}

template <class T, int DH, int NQ, int WQ, int KW>
atspeed_status launch_attention(const TreeAttnArgs& p, hipStream_t st) {
  const long long pairs = (long long)p.B * p.KH, n = (pairs + 7) / 8 * 8 * p.qtiles * p.splits;
  if (n >= (1LL << 31)) return fail(ATSPEED_E_SHAPE, "tree attention: too many query tiles");
  hipLaunchKernelGGL((tree_attn_kernel<T, DH, NQ, WQ, KW>), dim3((unsigned)n), dim3(256), 0, st, p);
  HIP_TRY(hipGetLastError());
  if (p.splits > 1) {
    const long long rows = (long long)p.B * p.max_new * p.H, per = 256 / (DH / 4);
    hipLaunchKernelGGL((tree_attn_join_kernel<T, DH>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, p);
    HIP_TRY(hipGetLastError());
  }
  return ATSPEED_OK;
}

template <class T, int DH>
atspeed_status run_attention(const TreeAttnArgs& p, int tile, hipStream_t st) {
  constexpr int KW1 = sizeof(T) == 2 ? 32 : 16;
  if (tile == 16) return launch_attention<T, DH, 1, 1, KW1>(p, st);
  if (tile == 32) return launch_attention<T, DH, 2, 1, KW1>(p, st);
  if (tile == 64) return launch_attention<T, DH, 1, 4, 64>(p, st);
  return launch_attention<T, DH, 2, 4, 64>(p, st);
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
  p.k = pages_dev(a.k_pages, es); p.v = pages_dev(a.v_pages, es);
  p.table = a.block_table; p.row_off = a.row_off; p.ctx = a.ctx; p.mask = a.mask;
  p.out = (char*)a.out; p.o_row = a.out_row_stride * es; p.o_head = a.out_head_stride * es;
  p.lse = a.lse;
  p.part = (float*)workspace; p.part_ml = (float2*)((char*)workspace + plan.part_bytes);
  p.B = a.B; p.n_rows = a.n_rows; p.H = a.n_heads; p.KH = a.n_kv_heads; p.G = a.n_heads / a.n_kv_heads;
  p.max_pages = a.max_pages; p.n_pool = a.n_pool; p.max_new = std::min(a.max_new, a.n_rows); p.words = a.mask_words;
  p.shift = log2_of(a.page_size); p.tail = a.page_size - 1;
  p.qtiles = plan.qtiles; p.splits = plan.splits; p.chunk = plan.chunk;
  // the queries carry the scale's sign, so that the largest product is the largest score
  p.q_flip = a.scale < 0.f ? (es == 2 ? 0x80008000u : 0x80000000u) : 0u;
  p.scale = std::max(std::fabs(a.scale) * 1.4426950408889634f, 1e-37f);
  hipStream_t st = (hipStream_t)stream;
  if (es == 2) return a.d_head == 64 ? run_attention<bf16_t, 64>(p, plan.tile, st) : run_attention<bf16_t, 128>(p, plan.tile, st);
  if (a.d_head == 32) return run_attention<float, 32>(p, plan.tile, st);
  if (a.d_head == 64) return run_attention<float, 64>(p, plan.tile, st);
  return run_attention<float, 128>(p, plan.tile, st);
}

}  // extern "C"
