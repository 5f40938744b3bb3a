// cache_append.hip -- new tokens into the paged int8 cache: queries and keys
// rotated by position, every value requantized to int8 with the scale of its
// query head, or of its page and kv head.
//
// Rotated values are exact integers in Q14 (|x| <= 128, cosines in Q14: below
// 2^23).  A scale S = max(1, ceil(A / 127)) comes from the largest magnitude A,
// so every code floor((2 r + S) / (2 S)) lies in [-127, 127], and with N = 2 r +
// 257 S the code + 128 is floor(N / (2 S)), 0 < N < 512 S.  With lg = ceil(log2
// S) and m = floor(2^(26 + lg) / (2 S)) + 1 that is floor(N m / 2^(26 + lg)):
// the excess N (2 S m - 2^(26 + lg)) <= 512 S 2 S <= 2^(10 + 2 lg) stays within
// 2^(26 + lg) for S <= 2^16.  Scaled to a common 2^48 the code is one byte of
// the product's high word: a shift, a 64-bit multiply-add and the byte permutes
// of the packing.
//
// Bound: one round trip through memory after the other (a few tokens: 3.8 us of one
// sequence, 5.3 of 64), bytes and the registers that keep them in flight (a prompt
// of 16384 tokens, 32 + 8 heads of 128: 41 us for the 31 that its 144 MB take to
// copy).  A team of threads, a wave for a few tokens and two for many, takes the
// new rows of a (page, kv head), keys and values apart; the queries are groups of
// D / 16 threads that take a head of 16-channel units each, and several heads of a
// token one after another so that its cosines are loaded once.
#include "decoder_internal.h"

namespace ilw {
namespace {


// Code bytes of values at scale S; see the top of the file.
struct Codes {
  int32_t S, sh, m2;
  int64_t c;
  __device__ __forceinline__ void init(int32_t s) {
    S = s;
    const int32_t lg = s > 1 ? 32 - __clz(s - 1) : 0;
    // The quotient is below 2^27 and no integer comes within 2^-17 above it: one
    // Newton step on the hardware's reciprocal (26 bits, then past 50) has its
    // floor.  Where it is an integer itself (S = 2^lg) one below gives m = the
    // quotient, no excess at all, and the same codes.
    const double d = (double)s, r = __builtin_amdgcn_rcp(d);
    const int32_t m = (int32_t)(__builtin_fma(__builtin_fma(-d, r, 1.0), r, r) *
                                (double)(1u << (25 + lg - 10)) * 1024.0) + 1;
    sh = 22 - lg;
    m2 = 2 * m;
    c = ((int64_t)257 * s * m) << sh;
  }
  // the high word whose byte 2 is code + 128
  __device__ __forceinline__ uint32_t word(int32_t r) const {
    return (uint32_t)(((int64_t)(int32_t)((uint32_t)r << sh) * m2 + c) >> 32);
  }
  __device__ __forceinline__ uint32_t pack(int32_t a, int32_t b, int32_t c2, int32_t d) const {
    const uint32_t lo = __builtin_amdgcn_perm(word(b), word(a), 0x0c0c0602u);
    const uint32_t hi = __builtin_amdgcn_perm(word(d), word(c2), 0x0c0c0602u);
    return (lo | (hi << 16)) ^ 0x80808080u;
  }
};

__device__ __forceinline__ int32_t byte_of(uint32_t w, int i) { return (int8_t)(w >> (8 * i)); }
__device__ __forceinline__ int32_t scale_for(uint32_t big) { return max(1, (int32_t)((big + 126) / 127)); }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 16 channels of a head: units 0 .. R/16 - 1 hold rotated pairs, 8 channels
// from `a` and the 8 from `b` that they pair with (or 16 consecutive channels,
// pairs interleaved), later units 16 consecutive channels that keep their value.
struct Unit {
  int32_t a, b;
  bool rot;
  __device__ __forceinline__ Unit(int i, int32_t R, bool inter) {
    rot = i * 16 < R;
    const bool split = rot && !inter;
    a = split ? i * 8 : i * 16;
    b = split ? i * 8 + R / 2 : i * 16 + 8;
  }
};

// The unit's cosines and sines at a position: 8 pairs, one word each.
__device__ __forceinline__ void load_rope(const int16_t* rope, int64_t pos, int32_t R, int i,
                                          v4i (&cs)[2]) {
  const v4i* p = (const v4i*)(rope + pos * R + i * 16);
  cs[0] = p[0];
  cs[1] = p[1];
}

template <bool INTER>
__device__ __forceinline__ void rotate(const u32x2& xa, const u32x2& xb, const v4i (&cs)[2],
                                       int32_t (&r)[16]) {
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int32_t w = cs[p >> 2][p & 3], co = (int16_t)w, si = w >> 16;
    // pair p: channels (a + p, b + p), or 2 p and 2 p + 1 of the 16
    const int i1 = INTER ? 2 * p : p, i2 = INTER ? 2 * p + 1 : p + 8;
    const int32_t x1 = byte_of(i1 < 8 ? xa[i1 >> 2] : xb[(i1 - 8) >> 2], i1 & 3);
    const int32_t x2 = byte_of(i2 < 8 ? xa[i2 >> 2] : xb[(i2 - 8) >> 2], i2 & 3);
    r[i1] = __mul24(x1, co) - __mul24(x2, si);
    r[i2] = __mul24(x2, co) + __mul24(x1, si);
  }
}

__device__ __forceinline__ void unit_values(const u32x2& xa, const u32x2& xb, const v4i (&cs)[2],
                                            bool rot, bool inter, int32_t (&r)[16]) {
  if (!rot) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      r[i] = (int32_t)((uint32_t)byte_of(i < 8 ? xa[i >> 2] : xb[(i - 8) >> 2], i & 3) << 14);
  } else if (inter) {
    rotate<true>(xa, xb, cs, r);
  } else {
    rotate<false>(xa, xb, cs, r);
  }
}

__device__ __forceinline__ uint32_t largest(const int32_t (&r)[16], uint32_t big) {
  int32_t hi = 0, lo = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    hi = max(hi, r[i]);
    lo = min(lo, r[i]);
  }
  return max(big, max((uint32_t)hi, (uint32_t)-lo));
}

// A sequence's new rows and where they start, whatever cu and past hold.
struct Rows {
  int32_t first, n, past;
  __device__ __forceinline__ Rows(const AppendArgs& a, int32_t s) {
    first = min(max(a.cu[s], 0), a.T);
    n = min(min(max(a.cu[s + 1], first), a.T) - first, a.max_new);
    past = min(max(a.past[s], 0), 1 << 21);
  }
};

// Threads of a team of TS: a wave or the whole workgroup.
template <int TS>
__device__ __forceinline__ uint32_t team_max(uint32_t v, uint32_t* lds) {
  v = (uint32_t)wave_max_i32((int32_t)v);  // below 2^31
  if constexpr (TS > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TS / 64; ++w) v = max(v, lds[w]);
  }
  return v;
}

// The largest of a group of n = 2, 4, 8 or 16 threads (halves that mirror each
// other: a mirror serves where an exchange would).
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t group_max(uint32_t v, int n) {
  v = max_with<0xb1>(v);              // quad_perm 1 0 3 2
  if (n > 2) v = max_with<0x4e>(v);   // quad_perm 2 3 0 1
  if (n > 4) v = max_with<0x141>(v);  // row_half_mirror
  if (n > 8) v = max_with<0x140>(v);  // row_mirror
  return v;
}

// The page's new scale, from the largest new value and the scale it had.
__device__ __forceinline__ int32_t page_scale(uint32_t big, bool fresh, int32_t old) {
  const int32_t need = scale_for(big);
  if (fresh) return need;
  return need <= old ? old : max(need, old + (old >> 3));
}

// What a team adds to one page and kv head: the new rows lo .. hi - 1 (tokens of
// the sequence), into the page's slots from lo - start on.
struct Part {
  int32_t block, start, lo, hi;
  __device__ __forceinline__ bool fresh() const { return lo == start; }
};

__device__ __forceinline__ bool page_of(const AppendArgs& a, int32_t s, const Part& p,
                                        int32_t& page) {
  page = a.c.table[(int64_t)s * a.c.max_pages + p.block];
  return (uint32_t)page < (uint32_t)a.c.n_pages;
}

// Two passes over the units, for the scale and with it, in opposite directions:
// the unit held last is used first, and with one unit a thread (a few tokens)
// nothing is read twice.  (Holding 2 or 4 units saves no time: 43 and 59 us a prompt
// against 42, nor does holding the cosines: 48.  Both cost registers, of which the
// kernel takes 85, five waves a SIMD.)
template <int TS>
__device__ void append_keys(const AppendArgs& a, const Rows& r, int32_t s, const Part& p,
                            int32_t h, int tid, uint32_t* lds) {
  const int32_t D = a.c.D, upr = D / 16, units = (p.hi - p.lo) * upr;
  const int8_t* src = a.qkv + (int64_t)(a.Hq + h) * D + (int64_t)(r.first - r.past) * a.ld;
  u32x2 xa, xb;
  // unit u: 16 channels of token lo + u / upr
  auto load = [&](int base) {
    const int u = base + tid;
    if (u >= units) return;
    const int32_t j = p.lo + u / upr, i = u % upr;
    const Unit un(i, a.R, a.inter);
    const int8_t* row = src + (int64_t)j * a.ld;
    xa = *(const u32x2*)(row + un.a);
    xb = *(const u32x2*)(row + un.b);
  };
  auto each = [&](int base, auto f) {
    const int u = base + tid;
    if (u >= units) return;
    const Unit un(u % upr, a.R, a.inter);
    int32_t v[16];
    v4i cs[2] = {};
    if (un.rot) load_rope(a.rope, p.lo + u / upr, a.R, u % upr, cs);
    unit_values(xa, xb, cs, un.rot, a.inter, v);
    f(p.lo + u / upr, un, v);
  };
  load(0);
  int32_t page;
  if (!page_of(a, s, p, page)) return;  // (the whole team)
  int8_t* dst = a.c.k + ((((int64_t)page * a.c.Hkv + h) << a.c.lp)) * D;
  // (read ahead of the barrier, after which the scale may be written)
  int32_t* scale = a.c.k_scale + (int64_t)page * a.c.Hkv + h;
  const int32_t old = p.fresh() ? 1 : min(max(*scale, 1), 1 << 16);
  uint32_t big = 0;
  auto find = [&](int32_t, const Unit&, int32_t(&v)[16]) { big = largest(v, big); };
  int base = 0;
  each(base, find);
  while (base + TS < units) {
    base += TS;
    load(base);
    each(base, find);
  }
  big = team_max<TS>(big, lds);
  const int32_t S = page_scale(big, p.fresh(), old);
  Codes q;
  q.init(S);
  if (S != old && !p.fresh()) {
    // (16 codes a step; the rows of a page are consecutive)
    for (int u = tid; u < (p.lo - p.start) * upr; u += TS) {
      v4i w = *(const v4i*)(dst + u * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = (int)q.pack(byte_of(w[i], 0) * old, byte_of(w[i], 1) * old, byte_of(w[i], 2) * old,
                           byte_of(w[i], 3) * old);
      *(v4i*)(dst + u * 16) = w;
    }
  }
  for (;;) {
    each(base, [&](int32_t j, const Unit& un, int32_t(&v)[16]) {
      int8_t* row = dst + (int64_t)(j - p.start) * D;
      *(u32x2*)(row + un.a) = u32x2{q.pack(v[0], v[1], v[2], v[3]), q.pack(v[4], v[5], v[6], v[7])};
      *(u32x2*)(row + un.b) =
          u32x2{q.pack(v[8], v[9], v[10], v[11]), q.pack(v[12], v[13], v[14], v[15])};
    });
    if (base == 0) break;
    base -= TS;
    load(base);
  }
  if (tid == 0) *scale = S;
}

// The same of the values, which lie as words of 4 tokens of a channel, for a few
// tokens by one wave.  A step takes 4 tokens of 4 channels.
__device__ void append_few_values(const AppendArgs& a, const Rows& r, int32_t s, const Part& p,
                                  int32_t h, int tid) {
  constexpr int TS = 64;
  const int32_t start = p.start, lo = p.lo, hi = p.hi;
  int32_t page;
  if (!page_of(a, s, p, page)) return;  // (the whole wave)
  const int32_t D = a.c.D, wpr = D / 4, P = 1 << a.c.lp, G = min(P, 64);
  const int8_t* src = a.qkv + (int64_t)(a.Hq + a.c.Hkv + h) * D +
                      (int64_t)(r.first - r.past) * a.ld;
  int8_t* dst = a.c.v + ((((int64_t)page * a.c.Hkv + h) << a.c.lp)) * D;
  int32_t* scale = a.c.v_scale + (int64_t)page * a.c.Hkv + h;
  const bool fresh = p.fresh();
  const int32_t old = fresh ? 1 : min(max(*scale, 1), 1 << 16);
  uint32_t big = 0;
  for (int u = tid; u < (hi - lo) * wpr; u += TS) {
    const int32_t j = lo + u / wpr;
    const uint32_t w = *(const uint32_t*)(src + (int64_t)j * a.ld + (u % wpr) * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) big = max(big, (uint32_t)abs(byte_of(w, i)));
  }
  big = team_max<TS>(big << 14, nullptr);
  const int32_t S = page_scale(big, fresh, old);
  const bool grown = S != old && !fresh;
  Codes q;
  q.init(S);
  const int32_t f = lo - start, l = hi - start;  // the new slots f .. l - 1
  const int32_t b0 = grown ? 0 : f / 4;
  for (int u = tid; u < ((l + 3) / 4 - b0) * wpr; u += TS) {
    const int32_t s0 = (b0 + u / wpr) * 4, c = (u % wpr) * 4, j = s0 % G;
    int8_t* at = dst + (s0 - j) * D + (c / 16) * 16 * G + ((j % 16) / 4) * 4 * G +
                 (c % 16) * (G / 4) + (j / 16) * 4;
    uint32_t x[4];  // 4 channels of each token
#pragma unroll
    for (int t = 0; t < 4; ++t)
      x[t] = s0 + t >= f && s0 + t < l
                 ? *(const uint32_t*)(src + (int64_t)(start + s0 + t) * a.ld + c)
                 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t* p = (uint32_t*)(at + i * (G / 4));
      uint32_t w = q.pack((int32_t)((uint32_t)byte_of(x[0], i) << 14),
                          (int32_t)((uint32_t)byte_of(x[1], i) << 14),
                          (int32_t)((uint32_t)byte_of(x[2], i) << 14),
                          (int32_t)((uint32_t)byte_of(x[3], i) << 14));
      if (s0 < f || s0 + 4 > l) {
        // tokens outside the new ones stay, at the new scale where it grew
        const uint32_t was = *p;
        uint32_t keep = was;
        if (grown)
          keep = q.pack(byte_of(was, 0) * old, byte_of(was, 1) * old, byte_of(was, 2) * old,
                        byte_of(was, 3) * old);
        uint32_t res = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t m = 0xffu << (8 * t);
          res |= m & (s0 + t < f ? keep : s0 + t < l ? w : was);
        }
        w = res;
      }
      *p = w;
    }
  }
  if (tid == 0) *scale = S;
}

// Values of many tokens.  A unit is what 4 channels hold of the tokens j, j + 16,
// ... of a group that share their j % 16 / 4: M words of 4 tokens of a channel,
// which lie one after another, and the 4 channels' words do too.  (Units of one
// word of each channel: every store 64 pieces of 4 bytes, 35 us of values of
// 16384 tokens and 8 kv heads of 128 against 17.)
template <int TS>
__device__ void append_values(const AppendArgs& a, const Rows& r, int32_t s, const Part& p,
                              int32_t h, int tid, uint32_t* lds) {
  const int32_t D = a.c.D, wpr = D / 4, P = 1 << a.c.lp, G = min(P, 64), M = G / 16;
  const int8_t* src = a.qkv + (int64_t)(a.Hq + a.c.Hkv + h) * D +
                      (int64_t)(r.first - r.past + p.start) * a.ld;
  const int32_t f = p.lo - p.start, l = p.hi - p.start;  // the new slots f .. l - 1
  const int32_t g0 = f / G, units = ((l + G - 1) / G - g0) * 4 * wpr;
  // first slot and channel of a unit, its place in the page
  struct Place {
    int32_t s0, c, at;
  };
  auto place = [&](int32_t g, int32_t u) {
    const int32_t jq = u / wpr, c = (u - jq * wpr) * 4;
    return Place{g * G + jq * 4, c,
                 g * G * D + (c / 16) * 16 * G + jq * 4 * G + (c % 16) * (G / 4)};
  };
  auto unit = [&](int u) {
    const int32_t g = u / (4 * wpr);
    return place(g0 + g, u - g * 4 * wpr);
  };
  uint32_t x[4][4];  // 4 channels of each token
  auto load = [&](int base) {
    const Place q = unit(base + tid);
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int32_t slot = q.s0 + 16 * m + t;
        x[m][t] = m < M && base + tid < units && slot >= f && slot < l
                      ? *(const uint32_t*)(src + (int64_t)slot * a.ld + q.c)
                      : 0;
      }
  };
  load(0);
  int32_t page;
  if (!page_of(a, s, p, page)) return;  // (the whole team)
  int8_t* dst = a.c.v + ((((int64_t)page * a.c.Hkv + h) << a.c.lp)) * D;
  int32_t* scale = a.c.v_scale + (int64_t)page * a.c.Hkv + h;
  const int32_t old = p.fresh() ? 1 : min(max(*scale, 1), 1 << 16);
  int32_t hi = 0, lo = 0;
  auto find = [&] {
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi = max(hi, byte_of(x[k / 4][k % 4], i));
        lo = min(lo, byte_of(x[k / 4][k % 4], i));
      }
  };
  int base = 0;
  find();
  while (base + TS < units) {
    base += TS;
    load(base);
    find();
  }
  const uint32_t big = team_max<TS>((uint32_t)max(hi, -lo) << 14, lds);
  const int32_t S = page_scale(big, p.fresh(), old);
  const bool grown = S != old && !p.fresh();
  Codes q;
  q.init(S);
  auto requant = [&](uint32_t w) {
    return q.pack(byte_of(w, 0) * old, byte_of(w, 1) * old, byte_of(w, 2) * old,
                  byte_of(w, 3) * old);
  };
  if (grown) {  // the groups before the new tokens' first
    for (int u = tid; u < g0 * G * wpr; u += TS) {
      uint32_t* w = (uint32_t*)dst + u;
      *w = requant(*w);
    }
  }
  for (;;) {
    if (base + tid < units) {
      const Place o = unit(base + tid);
      int8_t* to = dst + o.at;
      const bool whole = o.s0 >= f && o.s0 + G - 12 <= l;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int m = 0; m < 4; ++m)
          w[m] = q.pack((int32_t)((uint32_t)byte_of(x[m][0], i) << 14),
                        (int32_t)((uint32_t)byte_of(x[m][1], i) << 14),
                        (int32_t)((uint32_t)byte_of(x[m][2], i) << 14),
                        (int32_t)((uint32_t)byte_of(x[m][3], i) << 14));
        uint32_t* d = (uint32_t*)(to + i * (G / 4));
        if (whole && M == 4) {
          *(v4i*)d = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
          continue;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int32_t s0 = o.s0 + 16 * m;
          // words without new tokens change only where the scale grew, and only
          // in tokens before the new ones
          if (m >= M || s0 >= l || (s0 + 4 <= f && !grown)) continue;
          uint32_t v = w[m];
          if (s0 < f || s0 + 4 > l) {
            const uint32_t was = d[m], keep = grown ? requant(was) : was;
            v = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t)
              v |= 0xffu << (8 * t) & (s0 + t < f ? keep : s0 + t < l ? w[m] : was);
          }
          d[m] = v;
        }
      }
    }
    if (base == 0) break;
    base -= TS;
    load(base);
  }
  if (tid == 0) *scale = S;
}

// Blocks 0 .. kv_blocks - 1: teams of TS threads, one for each (sequence, page
// of those it may write, kv head, keys or values).  The others: the queries.
template <int TS, int NT>
__global__ __launch_bounds__(NT) void append_kernel(AppendArgs a, uint32_t nb, uint32_t kv_units,
                                                    uint32_t kv_blocks, int32_t hpu,
                                                    uint32_t q_blocks) {
  __shared__ uint32_t lds[NT / 64];
  if (blockIdx.x < kv_blocks) {
    const uint32_t unit = blockIdx.x * (NT / TS) +
                          (TS == 64 ? (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0u);
    if (unit >= kv_units) return;  // (whole teams)
    const uint32_t heads = 2 * (uint32_t)a.c.Hkv, sb = unit / heads, hv = unit - sb * heads;
    const int32_t s = (int32_t)(sb / nb), b = (int32_t)(sb - (uint32_t)s * nb);
    const Rows r(a, s);
    Part p;
    p.block = (r.past >> a.c.lp) + b;
    p.start = p.block << a.c.lp;
    p.lo = max(r.past, p.start);
    p.hi = min(r.past + r.n, p.start + (1 << a.c.lp));
    if (p.lo >= p.hi || p.block >= a.c.max_pages) return;
    const int tid = threadIdx.x % TS;
    const int32_t h = (int32_t)(hv >> 1);
    if (!(hv & 1)) append_keys<TS>(a, r, s, p, h, tid, lds);
    else if constexpr (TS == 64) append_few_values(a, r, s, p, h, tid);
    else append_values<TS>(a, r, s, p, h, tid, lds);
    return;
  }
  // queries: a group of D / 16 threads takes hpu heads of one token
  const int32_t D = a.c.D, upr = D / 16, groups = (a.Hq + hpu - 1) / hpu;
  const uint32_t qb = blockIdx.x - kv_blocks;
  const int32_t s = (int32_t)(qb / q_blocks);
  const uint32_t at = (qb - (uint32_t)s * q_blocks) * (NT / upr) + threadIdx.x / upr;
  const int32_t i = (int32_t)(at / (uint32_t)groups), h0 = (int32_t)(at - (uint32_t)i * groups) * hpu;
  const Rows r(a, s);
  if (i >= r.n) return;  // (whole groups of threads; they only talk among themselves)
  const int un_i = threadIdx.x % upr;
  const Unit un(un_i, a.R, a.inter);
  const int64_t t = r.first + i;
  const int32_t pos = min(r.past + i, (a.c.max_pages << a.c.lp) - 1);  // a row that rope has
  const int8_t* row = a.qkv + t * a.ld;
  v4i cs[2] = {};
  if (un.rot) load_rope(a.rope, pos, a.R, un_i, cs);
  const int32_t h1 = min(h0 + hpu, a.Hq);
  u32x2 na = *(const u32x2*)(row + h0 * D + un.a), nb2 = *(const u32x2*)(row + h0 * D + un.b);
  for (int32_t h = h0; h < h1; ++h) {
    const u32x2 xa = na, xb = nb2;
    if (h + 1 < h1) {  // the next head's, while this one is worked on
      na = *(const u32x2*)(row + (h + 1) * D + un.a);
      nb2 = *(const u32x2*)(row + (h + 1) * D + un.b);
    }
    int32_t v[16];
    unit_values(xa, xb, cs, un.rot, a.inter, v);
    uint32_t big = largest(v, 0);
    big = group_max(big, upr);
    Codes q;
    q.init(scale_for(big));
    int8_t* dst = a.q + (t * a.Hq + h) * D;
    *(u32x2*)(dst + un.a) = u32x2{q.pack(v[0], v[1], v[2], v[3]), q.pack(v[4], v[5], v[6], v[7])};
    *(u32x2*)(dst + un.b) =
        u32x2{q.pack(v[8], v[9], v[10], v[11]), q.pack(v[12], v[13], v[14], v[15])};
    if (un_i == 0) a.q_scale[t * a.Hq + h] = q.S;
  }
}

}  // namespace

namespace {

struct Grid {
  bool few;
  int32_t hpu, NT;
  int64_t nb, units, kv_blocks, q_blocks, total;
  explicit Grid(const AppendArgs& a) {
    const int32_t P = 1 << a.c.lp;
    // pages that max_new tokens can reach, whatever slot the first one takes
    nb = ((int64_t)a.max_new + P - 2) / P + 1;
    if (nb > a.c.max_pages) nb = a.c.max_pages;
    units = nb * a.seqs * 2 * a.c.Hkv;
    few = a.max_new <= 8;
    kv_blocks = few ? (units + 3) / 4 : units;
    hpu = few ? 1 : 8;
    NT = few ? 256 : 128;
    const int32_t groups = (a.Hq + hpu - 1) / hpu, per = NT / (a.c.D / 16);
    q_blocks = ((int64_t)a.max_new * groups + per - 1) / per;
    total = kv_blocks + q_blocks * a.seqs;
  }
};

}  // namespace

bool cache_append_fits(const AppendArgs& a) { return Grid(a).total < ((int64_t)1 << 24); }

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
  const Grid g(a);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)g.total), dim3(g.NT), 0, s, a, (uint32_t)g.nb,
                       (uint32_t)g.units, (uint32_t)g.kv_blocks, g.hpu, (uint32_t)g.q_blocks);
    return hipGetLastError();
  };
  return g.few ? launch(append_kernel<64, 256>) : launch(append_kernel<128, 128>);
}

}  // namespace ilw
