// cache_attention.hip -- integer attention over the paged int8 cache.
//
//   s = Q K^T (MFMA int8), rescaled to 1/64 octave by one 64-bit multiply-add
//   w = 2^(16 - (max s - s) / 64) by its chord, L = sum w
//   T = sum v p, p = w * value scale (15 bits, two int8 digits: MFMA int8 twice)
//   out = T / L requantized
//
// Queries that share a kv head are the rows of one product: row r of a sequence
// is query r / G of it and head r % G of the G heads.
//
// The chord of 2^x at x = n + f/64 is 2^n (1 + f/64), which is what the bits of a
// float with that exponent and those leading mantissa bits say: one shift-add of
// the score difference and a conversion to an integer (which floors) make w.
//
// The sums need the exact maximum first (a weight floored at one reference is not
// the shift of the weight floored at another), so the scores are made twice: once
// for the maximum, once for the weights.
#include "ilw_internal.h"

namespace ilw {
namespace {

constexpr int32_t kNone = -32768;   // below every score
constexpr int32_t kFar = 17 * 64;   // from here on a weight is 0

// A sequence's queries and keys, whatever cu and lens hold.
struct Seq {
  int32_t first, n, nq, len, end0;  // end0: one past the last key query 0 sees
  __device__ __forceinline__ Seq(const CacheAttnArgs& a, int32_t s) {
    first = min(max(a.cu[s], 0), a.T);
    n = min(max(a.cu[s + 1], first), a.T) - first;
    nq = min(n, a.max_q);
    const int32_t l = min(max(a.lens[s], 0), 1 << 20);
    len = min(l, a.max_len);
    end0 = a.causal ? l - n + 1 : l;
  }
};

// The keys a row sees: lo .. hi - 1.
struct Span {
  int32_t lo, hi;
  __device__ __forceinline__ Span(const CacheAttnArgs& a, const Seq& q, int32_t i) {
    const int32_t end = q.end0 + (a.causal ? i : 0);
    hi = min(max(end, 0), q.len);
    lo = a.window ? min(max(end - a.window, 0), hi) : 0;
  }
};

// The pages of 64 consecutive keys from key kb (a multiple of 64) on: one page,
// or two or four.  GB: 16-key blocks of a page among them.  numbers() then
// scales(): the second loads what the first one names.
template <int GB>
struct Pages {
  static constexpr int N = 4 / GB;
  int32_t page[N], ks[N], vs[N];
  bool ok;  // every page is there
  __device__ __forceinline__ void numbers(const CacheView& c, const int32_t* table, int32_t kb) {
#pragma unroll
    for (int i = 0; i < N; ++i) page[i] = table[min((kb >> c.lp) + i, c.max_pages - 1)];
  }
  // Keys of a page that is not there are read from page 0, and marked by a
  // negative key scale.
  __device__ __forceinline__ void scales(const CacheView& c, int32_t h) {
    ok = true;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool there = (uint32_t)page[i] < (uint32_t)c.n_pages;
      page[i] = there ? page[i] : 0;
      const int64_t at = (int64_t)page[i] * c.Hkv + h;
      ks[i] = there ? c.k_scale[at] : -1;
      vs[i] = c.v_scale[at];
      ok = ok && there;
    }
  }
  // byte offset of slot 0 of 16-key block u's page and head, and the block's slot
  __device__ __forceinline__ int64_t base(const CacheView& c, int32_t h, int u) const {
    return (((int64_t)page[u / GB] * c.Hkv + h) << c.lp) * c.D;
  }
  __device__ __forceinline__ static int32_t slot(const CacheView& c, int32_t kb, int u) {
    return GB == 4 ? (kb & ((1 << c.lp) - 1)) + 16 * u : 16 * (u % GB);
  }
};

template <int D>
struct Keys {
  static constexpr int KC = (D + 63) / 64;
  v4i f[4][KC];
  template <int GB>
  __device__ __forceinline__ void load(const CacheView& c, const Pages<GB>& pg, int32_t h,
                                       int32_t kb, int lane) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int8_t* p = c.k + pg.base(c, h, u) +
                        (Pages<GB>::slot(c, kb, u) + (lane & 15)) * D + (lane >> 4) * 16;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        f[u][kc] = D >= 64 || lane < 32 ? *(const v4i*)(p + kc * 64) : v4i{0, 0, 0, 0};
    }
  }
};

// 64 keys' values of 16 channels: a lane's 16 bytes are channel lane % 16 of
// keys 16 u + 4 (lane / 16) + r at byte 4 u + r.
template <int D, int GB>
__device__ __forceinline__ v4i load_values(const CacheView& c, const Pages<GB>& pg, int32_t h,
                                           int32_t kb, int g, int lane) {
  v4i v;
  if constexpr (GB == 4) {
    v = *(const v4i*)(c.v + pg.base(c, h, 0) + Pages<GB>::slot(c, kb, 0) * D + g * 1024 + lane * 16);
  } else if constexpr (GB == 2) {
    typedef int v2i __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const v2i x = *(const v2i*)(c.v + pg.base(c, h, 2 * i) + g * 512 + lane * 8);
      v[2 * i] = x[0];
      v[2 * i + 1] = x[1];
    }
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = *(const int32_t*)(c.v + pg.base(c, h, u) + g * 256 + lane * 4);
  }
  return v;
}

// (acc m + c) >> 28, low word
__device__ __forceinline__ int32_t rescale(int32_t acc, int32_t m, int64_t c) {
  const int64_t p = (int64_t)acc * m + c;
  return (int32_t)__builtin_amdgcn_alignbit((uint32_t)(p >> 32), (uint32_t)p, 28);
}
// The multiplier of a row's products with the keys of a page.
__device__ __forceinline__ int32_t score_mult(int32_t A, int32_t ks) {
  return (int32_t)(((int64_t)A * ks + (1 << 15)) >> 16);
}

constexpr int64_t kRnd = (int64_t)1 << 27;
// Added to w * value scale: the rounding of p, and 128 so that the two upper bytes
// are p's digits, the lower one with its sign bit flipped.
constexpr uint32_t kDigits = (1u << 15) + (128u << 16);

__device__ __forceinline__ int32_t med3(int32_t v, int32_t lo, int32_t hi) {
  int32_t r;
  asm("v_med3_i32 %0, %1, %2, %3" : "=v"(r) : "v"(v), "v"(lo), "v"(hi));
  return r;
}

// w of -a in [-kFar, 0].
__device__ __forceinline__ uint32_t weight(int32_t na) {
  return (uint32_t)__builtin_bit_cast(float, ((uint32_t)na << 17) + (143u << 23));
}

// The two digits of p for four weights and a value scale, a byte each.
struct Digits {
  uint32_t hi, lo;
  __device__ __forceinline__ Digits(const uint32_t (&w)[4], uint32_t vs) {
    uint32_t d[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) d[r] = __umul24(w[r], vs) + kDigits;
    const uint32_t d01 = __builtin_amdgcn_perm(d[1], d[0], 0x07030602u);
    const uint32_t d23 = __builtin_amdgcn_perm(d[3], d[2], 0x07030602u);
    lo = __builtin_amdgcn_perm(d23, d01, 0x05040100u) ^ 0x80808080u;
    hi = __builtin_amdgcn_perm(d23, d01, 0x07060302u);
  }
};

// Sum over the 4 lanes of a row.
__device__ __forceinline__ uint64_t sum_over_lanes(uint32_t v) {
  uint64_t l = (uint64_t)v + (uint32_t)__shfl_xor((int)v, 16, 64);
  const uint32_t l0 = __shfl_xor((int)(uint32_t)l, 32, 64), l1 = __shfl_xor((int)(l >> 32), 32, 64);
  return l + (((uint64_t)l1 << 32) | l0);
}

// One row's requantization of T: its weight sum's shift and factor.
struct Norm {
  uint32_t F;
  int32_t sh;
  __device__ __forceinline__ void init(uint64_t L) {
    const int32_t d = L ? 48 - __clzll((long long)L) : 1;  // bit length - 16 (L >= 2^16 or 0)
    F = L ? div_2p31m1((uint32_t)(L >> d)) : 0;
    sh = d + 13;
  }
  __device__ __forceinline__ int32_t out(int64_t T, int32_t mult, int32_t shift) const {
    const int32_t r = (int32_t)((T * (int64_t)F) >> sh);
    return rq(r, mult, shift);
  }
};

// A wave's 16 NF rows: a lane holds those of column lane % 16 of each fragment.
// Rows past the last one repeat it.
template <int D, int NF>
struct Rows {
  static constexpr int KC = Keys<D>::KC;
  int32_t A[NF], lo[NF], hi[NF];
  v4i q[NF][KC];
  int64_t at[NF];
  int32_t all_lo, all_hi, any_lo, any_hi;  // keys that all of them, or some, see
  __device__ __forceinline__ void load(const CacheAttnArgs& a, const Seq& sq, int32_t h, int32_t G,
                                       int32_t r0, int32_t rows, int lane) {
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int32_t r = min(r0 + f * 16 + (lane & 15), rows - 1), i = r / G, g = r - i * G;
      const Span sp(a, sq, i);
      lo[f] = sp.lo;
      hi[f] = sp.hi;
      at[f] = (int64_t)(sq.first + i) * a.Hq + h * G + g;
      A[f] = (int32_t)(((int64_t)a.q_scale[at[f]] * a.score_mult +
                        ((int64_t)1 << (a.score_t - 1))) >> a.score_t);
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        q[f][kc] = D >= 64 || lane < 32
                       ? *(const v4i*)(a.q + at[f] * D + kc * 64 + (lane >> 4) * 16)
                       : v4i{0, 0, 0, 0};
    }
    // (later rows see later keys)
    const Span s0(a, sq, r0 / G), s1(a, sq, (min(r0 + 16 * NF, rows) - 1) / G);
    any_lo = s0.lo;
    all_lo = s1.lo;
    all_hi = s0.hi;
    any_hi = s1.hi;
  }
  __device__ __forceinline__ bool sees(int f, int32_t key, int32_t ks) const {
    return key >= lo[f] && key < hi[f] && ks >= 0;
  }
  // products of 16-key block u
  __device__ __forceinline__ v4i products(const Keys<D>& k, int u, int f) const {
    v4i p = {0, 0, 0, 0};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
      p = __builtin_amdgcn_mfma_i32_16x16x64_i8(k.f[u][kc], q[f][kc], p, 0, 0, 0);
    return p;
  }
};

// A row's largest score once its lanes (and waves) agree: the reference of the
// weights, and the score difference from which on they are all alike (0, or that
// of the lowest score there is).
struct Ref {
  int64_t c;
  int32_t cap, m;
  __device__ __forceinline__ void init(int32_t top) {
    m = min(top, 32767);
    c = kRnd - (int64_t)m * (1 << 28);
    cap = -max(0, min(kFar, m + 32767));
  }
};

__device__ __forceinline__ int32_t over_lanes(int32_t m) {  // of a row
  m = max(m, __shfl_xor(m, 16, 64));
  return max(m, __shfl_xor(m, 32, 64));
}

// Many rows: 16 NF rows of a (sequence, kv head) over all their keys twice, by one
// wave.
template <int D, int GB, int NF>
__global__ __launch_bounds__(256) void cache_rows_kernel(CacheAttnArgs a, uint32_t tiles) {
  constexpr int CG = D / 16;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t pair = blockIdx.x / tiles, tile = tiles - 1 - (blockIdx.x - pair * tiles);
  const int32_t s = (int32_t)(pair / (uint32_t)a.c.Hkv), h = (int32_t)(pair - (uint32_t)s * a.c.Hkv);
  const int32_t G = a.Hq / a.c.Hkv;
  const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
  const Seq sq(a, s);
  const int32_t rows = sq.nq * G, r0 = ((int32_t)tile * 4 + wave) * 16 * NF;
  if (r0 >= rows) return;
  Rows<D, NF> R;
  R.load(a, sq, h, G, r0, rows, lane);
  const int32_t kb0 = R.any_lo & ~63, kend = R.any_hi;
  auto full = [&](int32_t kb) { return kb >= R.all_lo && kb + 64 <= R.all_hi; };
  const v4i zero = {0, 0, 0, 0};

  // ---- maxima.  The keys of the next step, and the page numbers of the one
  // after it, are on their way during a step (past the last one too: any page
  // number leads to a page).
  int32_t M[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) M[f] = kNone;
  {
    Pages<GB> p0, p1;
    Keys<D> k0;
    p0.numbers(a.c, table, kb0);
    p1.numbers(a.c, table, kb0 + 64);
    p0.scales(a.c, h);
    k0.load(a.c, p0, h, kb0, lane);
    for (int32_t kb = kb0; kb < kend; kb += 64) {
      Pages<GB> p2;
      Keys<D> k1;
      p2.numbers(a.c, table, kb + 128);
      p1.scales(a.c, h);
      k1.load(a.c, p1, h, kb + 64, lane);
      if (full(kb) && p0.ok) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            const v4i p = R.products(k0, u, f);
            M[f] = max(max(M[f], -32767), rescale(max(max(p[0], p[1]), max(p[2], p[3])),
                                                  score_mult(R.A[f], p0.ks[u / GB]), kRnd));
          }
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            const v4i p = R.products(k0, u, f);
            const int32_t m = score_mult(R.A[f], p0.ks[u / GB]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (R.sees(f, kb + 16 * u + 4 * (lane >> 4) + r, p0.ks[u / GB]))
                M[f] = max(max(M[f], -32767), rescale(p[r], m, kRnd));
          }
      }
      p0 = p1;
      p1 = p2;
      k0 = k1;
    }
  }
  Ref ref[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) ref[f].init(over_lanes(M[f]));

  // ---- weights and sums
  v4i oh[CG][NF], ol[CG][NF];
  uint32_t L[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    L[f] = 0;
#pragma unroll
    for (int g = 0; g < CG; ++g) oh[g][f] = ol[g][f] = zero;
  }
  {
    Pages<GB> p0, p1;
    Keys<D> k0;
    p0.numbers(a.c, table, kb0);
    p1.numbers(a.c, table, kb0 + 64);
    p0.scales(a.c, h);
    k0.load(a.c, p0, h, kb0, lane);
    for (int32_t kb = kb0; kb < kend; kb += 64) {
      Pages<GB> p2;
      p2.numbers(a.c, table, kb + 128);
      p1.scales(a.c, h);
      v4i vf[CG];
#pragma unroll
      for (int g = 0; g < CG; ++g) vf[g] = load_values<D, GB>(a.c, p0, h, kb, g, lane);
      v4i sc[4][NF];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int f = 0; f < NF; ++f) sc[u][f] = R.products(k0, u, f);
      k0.load(a.c, p1, h, kb + 64, lane);
      const bool fast = full(kb) && p0.ok;
      v4i ph[NF], pl[NF];
      auto weights = [&](auto checked) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            const int32_t m = score_mult(R.A[f], p0.ks[u / GB]);
            uint32_t w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              w[r] = weight(med3(rescale(sc[u][f][r], m, ref[f].c), ref[f].cap, 0));
              if (decltype(checked)::value &&
                  !R.sees(f, kb + 16 * u + 4 * (lane >> 4) + r, p0.ks[u / GB]))
                w[r] = 0;
            }
            L[f] += w[0] + w[1] + w[2] + w[3];
            const Digits d(w, (uint32_t)p0.vs[u / GB]);
            ph[f][u] = (int)d.hi;
            pl[f][u] = (int)d.lo;
          }
      };
      if (fast) weights(Flag<false>{});
      else weights(Flag<true>{});
#pragma unroll
      for (int g = 0; g < CG; ++g)
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          oh[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[g], ph[f], oh[g][f], 0, 0, 0);
          ol[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[g], pl[f], ol[g][f], 0, 0, 0);
        }
      p0 = p1;
      p1 = p2;
    }
  }
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    Norm nm;
    nm.init(sum_over_lanes(L[f]));
    if (r0 + f * 16 + (lane & 15) >= rows) continue;
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      int32_t v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[r] = nm.out((int64_t)oh[g][f][r] * 256 + ol[g][f][r], a.out_mult, a.out_shift);
      *(uint32_t*)(a.out + R.at[f] * D + g * 16 + (lane >> 4) * 4) = pack4(v[0], v[1], v[2], v[3]);
    }
  }
}

// ---- few rows (a tile of up to 16), many keys: the waves of a workgroup, and
// where that is not enough several workgroups, split the keys.  Scores, as 16-bit
// numbers (kNone: not seen), wait in LDS or in the workspace until the maximum is
// known; sums meet in LDS, partial ones in the workspace.
struct Split {
  int16_t* scores;  // [tiles][steps][rpt][64]; a row's 64 in the order of the lanes
  int32_t* top;     // [tiles][nsplit][16]
  int64_t* T;       // [tiles][nsplit][rpt][D]
  uint64_t* L;      // [tiles][nsplit][16]
  int32_t rt, rpt, steps, nsplit, chunk;  // row tiles a pair, rows a tile, keys a split
};

// The tile of a workgroup: its sequence, kv head and rows, and its chunks of keys.
struct Few {
  int32_t s, h, G, r0, rows, first, last;  // chunks first .. last - 1 hold keys
  __device__ __forceinline__ Few(const CacheAttnArgs& a, const Split& sp, uint32_t tile) {
    const uint32_t pair = tile / (uint32_t)sp.rt;
    s = (int32_t)(pair / (uint32_t)a.c.Hkv);
    h = (int32_t)(pair - (uint32_t)s * a.c.Hkv);
    G = a.Hq / a.c.Hkv;
    r0 = (int32_t)(tile - pair * (uint32_t)sp.rt) * 16;
  }
  __device__ __forceinline__ bool bounds(const CacheAttnArgs& a, const Split& sp, const Seq& sq) {
    rows = sq.nq * G;
    if (r0 >= rows) return false;
    const Span s0(a, sq, r0 / G), s1(a, sq, (min(r0 + 16, rows) - 1) / G);
    first = s0.lo / sp.chunk;
    last = s1.hi > s0.lo ? (s1.hi + sp.chunk - 1) / sp.chunk : first;
    return true;
  }
};

// Scores of the wave's steps (every NW-th from `wave` on) of keys c0 .. c1 - 1, to
// out(step, words); the row's maximum over them comes back.
template <int D, int GB, int NW, typename Out>
__device__ __forceinline__ int32_t few_scores(const CacheAttnArgs& a, const Rows<D, 1>& R,
                                              const int32_t* table, int32_t h, int32_t c0,
                                              int32_t c1, int wave, int lane, Out out) {
  int32_t M = kNone;
  const int32_t kb0 = c0 + wave * 64;
  if (kb0 >= c1) return M;
  Pages<GB> p0, p1;
  Keys<D> k0;
  p0.numbers(a.c, table, kb0);
  p1.numbers(a.c, table, kb0 + 64 * NW);
  p0.scales(a.c, h);
  k0.load(a.c, p0, h, kb0, lane);
  for (int32_t kb = kb0; kb < c1; kb += 64 * NW) {
    Pages<GB> p2;
    Keys<D> k1;
    p2.numbers(a.c, table, kb + 128 * NW);
    p1.scales(a.c, h);
    k1.load(a.c, p1, h, kb + 64 * NW, lane);
    const bool fast = kb >= R.all_lo && kb + 64 <= R.all_hi && p0.ok;
    v4i w[2];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const v4i p = R.products(k0, u, 0);
      const int32_t m = score_mult(R.A[0], p0.ks[u / GB]);
      int32_t x[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = med3(rescale(p[r], m, kRnd), -32767, 32767);
        if (!fast && !R.sees(0, kb + 16 * u + 4 * (lane >> 4) + r, p0.ks[u / GB])) x[r] = kNone;
        M = max(M, x[r]);
      }
#pragma unroll
      for (int r = 0; r < 2; ++r)
        w[u / 2][(u % 2) * 2 + r] = (int)__builtin_amdgcn_perm((uint32_t)x[2 * r + 1],
                                                               (uint32_t)x[2 * r], 0x05040100u);
    }
    out(kb >> 6, w);
    p0 = p1;
    p1 = p2;
    k0 = k1;
  }
  return M;
}

// Weights and sums of the same steps, the scores from in(step).
template <int D, int GB, int NW, typename In>
__device__ __forceinline__ uint32_t few_values(const CacheAttnArgs& a, const Ref& ref,
                                               const int32_t* table, int32_t h, int32_t c0,
                                               int32_t c1, int wave, int lane, In in,
                                               v4i (&oh)[D / 16], v4i (&ol)[D / 16]) {
  constexpr int CG = D / 16;
  uint32_t L = 0;
  const v4i zero = {0, 0, 0, 0};
#pragma unroll
  for (int g = 0; g < CG; ++g) oh[g] = ol[g] = zero;
  const int32_t kb0 = c0 + wave * 64;
  if (kb0 >= c1) return L;
  Pages<GB> p0, p1;
  v4i v0[CG];
  p0.numbers(a.c, table, kb0);
  p1.numbers(a.c, table, kb0 + 64 * NW);
  p0.scales(a.c, h);
#pragma unroll
  for (int g = 0; g < CG; ++g) v0[g] = load_values<D, GB>(a.c, p0, h, kb0, g, lane);
  for (int32_t kb = kb0; kb < c1; kb += 64 * NW) {
    Pages<GB> p2;
    v4i v1[CG], x[2], ph, pl;
    in(kb >> 6, x);
    p2.numbers(a.c, table, kb + 128 * NW);
    p1.scales(a.c, h);
#pragma unroll
    for (int g = 0; g < CG; ++g) v1[g] = load_values<D, GB>(a.c, p1, h, kb + 64 * NW, g, lane);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int32_t two = x[u / 2][(u % 2) * 2 + r / 2];
        const int32_t sc = r % 2 ? two >> 16 : (int16_t)two;
        w[r] = sc == kNone ? 0 : weight(med3(sc - ref.m, ref.cap, 0));
      }
      L += w[0] + w[1] + w[2] + w[3];
      const Digits d(w, (uint32_t)p0.vs[u / GB]);
      ph[u] = (int)d.hi;
      pl[u] = (int)d.lo;
    }
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      oh[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v0[g], ph, oh[g], 0, 0, 0);
      ol[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v0[g], pl, ol[g], 0, 0, 0);
    }
    p0 = p1;
    p1 = p2;
#pragma unroll
    for (int g = 0; g < CG; ++g) v0[g] = v1[g];
  }
  return L;
}

// The waves' sums added up in LDS (whole numbers: in any order); T of value
// channels 16 g + 4 (lane / 16) + r, row lane % 16, at word (g 64 + lane) 4 + r.
template <int D, int NW>
struct FewSums {
  int32_t hi[D / 16 * 256], lo[D / 16 * 256];
  unsigned long long L[16];
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < D / 16 * 256; i += 64 * NW) hi[i] = lo[i] = 0;
    if (threadIdx.x < 16) L[threadIdx.x] = 0;
  }
  __device__ __forceinline__ void add(uint32_t l, const v4i (&oh)[D / 16], const v4i (&ol)[D / 16],
                                      int32_t rows, int lane) {
    const uint64_t all = sum_over_lanes(l);
    if (lane < 16) atomicAdd(&L[lane], (unsigned long long)all);
    if ((lane & 15) >= rows) return;
#pragma unroll
    for (int g = 0; g < D / 16; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        atomicAdd(&hi[(g * 64 + lane) * 4 + r], oh[g][r]);
        atomicAdd(&lo[(g * 64 + lane) * 4 + r], ol[g][r]);
      }
  }
  __device__ __forceinline__ int64_t T(int i) const { return (int64_t)hi[i] * 256 + lo[i]; }
};

// One workgroup for all keys of a tile.
template <int D, int GB, int NW>
__global__ __launch_bounds__(64 * NW) void cache_few_kernel(CacheAttnArgs a, Split sp) {
  extern __shared__ __attribute__((aligned(16))) int8_t dyn[];  // scores [steps][rpt][64]
  __shared__ __attribute__((aligned(16))) FewSums<D, NW> sums;
  __shared__ int32_t top[NW][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Few t(a, sp, blockIdx.x);
  const int32_t* table = a.c.table + (int64_t)t.s * a.c.max_pages;
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq)) return;
  Rows<D, 1> R;
  R.load(a, sq, t.h, t.G, t.r0, t.rows, lane);
  const int32_t n = min(16, t.rows - t.r0), c0 = R.any_lo & ~63;
  int16_t* scores = (int16_t*)dyn + (lane >> 4) * 16 + (lane & 15) * 64;
  const int32_t stride = sp.rpt * 64, s0 = c0 >> 6;
  sums.clear();
  const int32_t M = over_lanes(few_scores<D, GB, NW>(
      a, R, table, t.h, c0, R.any_hi, wave, lane, [&](int32_t step, const v4i(&w)[2]) {
        if ((lane & 15) >= n) return;
        v4i* p = (v4i*)(scores + (step - s0) * stride);
        p[0] = w[0];
        p[1] = w[1];
      }));
  if (lane < 16) top[wave][lane] = M;
  lds_sync();
  int32_t m = kNone;
#pragma unroll
  for (int w = 0; w < NW; ++w) m = max(m, top[w][lane & 15]);
  Ref ref;
  ref.init(m);
  v4i oh[D / 16], ol[D / 16];
  const int32_t back = max((lane & 15) - (n - 1), 0) * 64;  // rows past the last repeat it
  const uint32_t L = few_values<D, GB, NW>(
      a, ref, table, t.h, c0, R.any_hi, wave, lane, [&](int32_t step, v4i(&x)[2]) {
        const v4i* p = (const v4i*)(scores + (step - s0) * stride - back);
        x[0] = p[0];
        x[1] = p[1];
      }, oh, ol);
  sums.add(L, oh, ol, n, lane);
  lds_sync();
  for (int i = threadIdx.x; i < D / 16 * 64; i += 64 * NW) {
    const int ln = i & 63, g = i >> 6, row = ln & 15;
    if (row >= n) continue;
    Norm nm;
    nm.init(sums.L[row]);
    int32_t v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = nm.out(sums.T(i * 4 + k), a.out_mult, a.out_shift);
    const int32_t r = t.r0 + row, q = r / t.G;
    *(uint32_t*)(a.out + ((int64_t)(sq.first + q) * a.Hq + t.h * t.G + r - q * t.G) * D + g * 16 +
                 (ln >> 4) * 4) = pack4(v[0], v[1], v[2], v[3]);
  }
}

// Several workgroups a tile, three launches: scores and maxima, sums, the output.
template <int D, int GB>
__global__ __launch_bounds__(256) void split_scores_kernel(CacheAttnArgs a, Split sp) {
  __shared__ int32_t top[4][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tile = blockIdx.x / (uint32_t)sp.nsplit;
  const int32_t part = (int32_t)(blockIdx.x - tile * (uint32_t)sp.nsplit);
  Few t(a, sp, tile);
  const int32_t* table = a.c.table + (int64_t)t.s * a.c.max_pages;
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq) || part < t.first || part >= t.last) return;
  Rows<D, 1> R;
  R.load(a, sq, t.h, t.G, t.r0, t.rows, lane);
  const int32_t n = min(16, t.rows - t.r0);
  const int32_t c0 = max(part * sp.chunk, R.any_lo & ~63), c1 = min((part + 1) * sp.chunk, R.any_hi);
  int16_t* scores = sp.scores + (int64_t)tile * sp.steps * sp.rpt * 64 + (lane >> 4) * 16 +
                    (lane & 15) * 64;
  const int32_t M = over_lanes(few_scores<D, GB, 4>(
      a, R, table, t.h, c0, c1, wave, lane, [&](int32_t step, const v4i(&w)[2]) {
        if ((lane & 15) >= n) return;
        v4i* p = (v4i*)(scores + (int64_t)step * sp.rpt * 64);
        p[0] = w[0];
        p[1] = w[1];
      }));
  if (lane < 16) top[wave][lane] = M;
  lds_sync();
  if (threadIdx.x < 16) {
    int32_t m = kNone;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = max(m, top[w][lane]);
    sp.top[((int64_t)tile * sp.nsplit + part) * 16 + lane] = m;
  }
}

template <int D, int GB>
__global__ __launch_bounds__(256) void split_values_kernel(CacheAttnArgs a, Split sp) {
  __shared__ __attribute__((aligned(16))) FewSums<D, 4> sums;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tile = blockIdx.x / (uint32_t)sp.nsplit;
  const int32_t part = (int32_t)(blockIdx.x - tile * (uint32_t)sp.nsplit);
  Few t(a, sp, tile);
  const int32_t* table = a.c.table + (int64_t)t.s * a.c.max_pages;
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq) || part < t.first || part >= t.last) return;
  const Span s0(a, sq, t.r0 / t.G), s1(a, sq, (min(t.r0 + 16, t.rows) - 1) / t.G);
  const int32_t n = min(16, t.rows - t.r0);
  const int32_t c0 = max(part * sp.chunk, s0.lo & ~63), c1 = min((part + 1) * sp.chunk, s1.hi);
  sums.clear();
  int32_t m = kNone;
  for (int32_t i = t.first + (lane >> 4); i < t.last; i += 4)
    m = max(m, sp.top[((int64_t)tile * sp.nsplit + i) * 16 + (lane & 15)]);
  Ref ref;
  ref.init(over_lanes(m));
  const int16_t* scores = sp.scores + (int64_t)tile * sp.steps * sp.rpt * 64 + (lane >> 4) * 16 +
                          min(lane & 15, n - 1) * 64;
  v4i oh[D / 16], ol[D / 16];
  const uint32_t L = few_values<D, GB, 4>(
      a, ref, table, t.h, c0, c1, wave, lane, [&](int32_t step, v4i(&x)[2]) {
        const v4i* p = (const v4i*)(scores + (int64_t)step * sp.rpt * 64);
        x[0] = p[0];
        x[1] = p[1];
      }, oh, ol);
  lds_sync();
  sums.add(L, oh, ol, n, lane);
  lds_sync();
  const int64_t at = (int64_t)tile * sp.nsplit + part;
  for (int i = threadIdx.x; i < D / 16 * 64; i += 256) {
    const int ln = i & 63, g = i >> 6, row = ln & 15;
    if (row >= n) continue;
    int64_t* dst = sp.T + (at * sp.rpt + row) * D + g * 16 + (ln >> 4) * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) dst[k] = sums.T(i * 4 + k);
  }
  if (threadIdx.x < 16) sp.L[at * 16 + threadIdx.x] = sums.L[threadIdx.x];
}

// A workgroup a row: D / 4 threads a part, 4 channels each.
template <int D>
__global__ __launch_bounds__(256) void split_join_kernel(CacheAttnArgs a, Split sp) {
  constexpr int Q = D / 4, PP = 256 / Q;  // channel quads, parts side by side
  __shared__ int64_t part_T[PP][D];
  __shared__ uint64_t part_L[PP];
  const uint32_t tile = blockIdx.x / (uint32_t)sp.rpt;
  const int32_t row = (int32_t)(blockIdx.x - tile * (uint32_t)sp.rpt);
  Few t(a, sp, tile);
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq) || t.r0 + row >= t.rows) return;
  const int q = threadIdx.x % Q, p0 = threadIdx.x / Q;
  int64_t T[4] = {0, 0, 0, 0};
  uint64_t L = 0;
#pragma unroll 4
  for (int32_t i = t.first + p0; i < t.last; i += PP) {
    const int64_t at = (int64_t)tile * sp.nsplit + i;
    const int64_t* src = sp.T + (at * sp.rpt + row) * D + q * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) T[k] += src[k];
    L += sp.L[at * 16 + row];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part_T[p0][q * 4 + k] = T[k];
  if (q == 0) part_L[p0] = L;
  lds_sync();
  if (threadIdx.x >= Q) return;
  L = 0;
  for (int i = 0; i < PP; ++i) L += part_L[i];
  Norm nm;
  nm.init(L);
  int32_t v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    int64_t x = 0;
    for (int i = 0; i < PP; ++i) x += part_T[i][q * 4 + k];
    v[k] = nm.out(x, a.out_mult, a.out_shift);
  }
  const int32_t r = t.r0 + row, i = r / t.G;
  *(uint32_t*)(a.out + ((int64_t)(sq.first + i) * a.Hq + t.h * t.G + r - i * t.G) * D + q * 4) =
      pack4(v[0], v[1], v[2], v[3]);
}

// ---- which kernels
enum Way { ROWS, FEW, SPLIT };
struct Plan {
  Way way;
  Split sp;
  int64_t tiles;
  size_t bytes;  // of the workspace
};
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

Plan plan(const CacheAttnArgs& a) {
  Plan p = {};
  const int64_t G = a.Hq / a.c.Hkv, rows = a.max_q * G, pairs = (int64_t)a.seqs * a.c.Hkv;
  p.sp.rt = (int32_t)((rows + 15) / 16);
  p.sp.rpt = (int32_t)(rows < 16 ? rows : 16);
  p.sp.steps = (a.max_len + 63) / 64;
  p.tiles = pairs * p.sp.rt;
  p.sp.nsplit = 1;
  p.sp.chunk = p.sp.steps * 64 + 64;
  if (p.tiles == 0 || p.sp.steps == 0) {
    p.way = FEW;
    return p;
  }
  if (rows > 64 && a.max_len <= 131072) {
    p.way = ROWS;
    return p;
  }
  const size_t lds = (size_t)p.sp.steps * p.sp.rpt * 128;
  if (a.max_len <= 1024 && lds <= 32768) {
    p.way = FEW;
    return p;
  }
  p.way = SPLIT;
  int64_t chunk = (a.max_len * p.tiles + 1023) / 1024;
  chunk = (chunk + 255) / 256 * 256;
  if (chunk < 512) chunk = 512;
  if (chunk > 32768) chunk = 32768;
  p.sp.chunk = (int32_t)chunk;
  p.sp.nsplit = (int32_t)((a.max_len + chunk - 1) / chunk);
  const int64_t parts = p.tiles * p.sp.nsplit;
  p.bytes = align256((size_t)p.tiles * p.sp.steps * p.sp.rpt * 128) + align256((size_t)parts * 64) +
            align256((size_t)parts * p.sp.rpt * a.c.D * 8) + align256((size_t)parts * 128);
  return p;
}

template <int D, int GB>
hipError_t launch_pages(const CacheAttnArgs& a, void* ws, hipStream_t s) {
  Plan p = plan(a);
  if (p.tiles == 0) return hipSuccess;
  if (p.way == ROWS) {
    constexpr int NF = D >= 256 ? 1 : 2;
    const int64_t rows = (int64_t)a.max_q * (a.Hq / a.c.Hkv);
    const uint32_t tiles = (uint32_t)((rows + 64 * NF - 1) / (64 * NF));
    const int64_t total = (int64_t)tiles * a.seqs * a.c.Hkv;
    if (total >= ((int64_t)1 << 24)) return hipErrorInvalidValue;  // under 2^32 threads
    hipLaunchKernelGGL((cache_rows_kernel<D, GB, NF>), dim3((unsigned)total), dim3(256), 0, s, a,
                       tiles);
    return hipGetLastError();
  }
  if (p.tiles * p.sp.nsplit >= ((int64_t)1 << 23) || p.tiles * 16 >= ((int64_t)1 << 24))
    return hipErrorInvalidValue;
  if (p.way == FEW) {
    constexpr int NW = 8;
    hipLaunchKernelGGL((cache_few_kernel<D, GB, NW>), dim3((unsigned)p.tiles), dim3(64 * NW),
                       (unsigned)(p.sp.steps * p.sp.rpt * 128), s, a, p.sp);
    return hipGetLastError();
  }
  const int64_t parts = p.tiles * p.sp.nsplit;
  int8_t* at = (int8_t*)ws;
  auto take = [&](size_t n) {
    int8_t* r = at;
    at += align256(n);
    return r;
  };
  p.sp.scores = (int16_t*)take((size_t)p.tiles * p.sp.steps * p.sp.rpt * 128);
  p.sp.top = (int32_t*)take((size_t)parts * 64);
  p.sp.T = (int64_t*)take((size_t)parts * p.sp.rpt * D * 8);
  p.sp.L = (uint64_t*)take((size_t)parts * 128);
  hipLaunchKernelGGL((split_scores_kernel<D, GB>), dim3((unsigned)parts), dim3(256), 0, s, a, p.sp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((split_values_kernel<D, GB>), dim3((unsigned)parts), dim3(256), 0, s, a, p.sp);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((split_join_kernel<D>), dim3((unsigned)(p.tiles * p.sp.rpt)), dim3(256), 0, s, a,
                     p.sp);
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const CacheAttnArgs& a, void* ws, hipStream_t s) {
  return a.c.lp >= 6 ? launch_pages<D, 4>(a, ws, s)
                     : a.c.lp == 5 ? launch_pages<D, 2>(a, ws, s) : launch_pages<D, 1>(a, ws, s);
}

}  // namespace

size_t cache_attention_workspace(const CacheAttnArgs& a) { return plan(a).bytes; }

hipError_t launch_cache_attention(const CacheAttnArgs& a, void* ws, hipStream_t s) {
  switch (a.c.D) {
    case 32: return launch_dim<32>(a, ws, s);
    case 64: return launch_dim<64>(a, ws, s);
    case 128: return launch_dim<128>(a, ws, s);
    default: return launch_dim<256>(a, ws, s);
  }
}

}  // namespace ilw
