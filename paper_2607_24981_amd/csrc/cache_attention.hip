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
#include "decoder_internal.h"

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
// or two or four.  GB: 16-key blocks of a page among them.  Keys of a page that is
// not there are read from page 0; a negative key scale marks them.
template <int GB>
struct Pages {
  static constexpr int N = 4 / GB;
  int32_t page[N], ks[N], vs[N];
  int32_t lanes, lane0;  // GB == 1: a page number a lane, the first page's lane
  __device__ __forceinline__ bool all() const {
    int32_t m = ks[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = min(m, ks[i]);
    return m >= 0;
  }
  // byte offset of slot 0 of 16-key block u's page and head, and the block's slot
  __device__ __forceinline__ int64_t base(const CacheView& c, int32_t h, int u) const {
    return (((int64_t)page[u / GB] * c.Hkv + h) << c.lp) * c.D;
  }
  // The same for a uniform block number that is not a constant: of one or two pages
  // by selects, of four from the lanes that hold them.  (Of four selects the compiler
  // made an array in memory, stored and loaded in every step: prompts of 4 x 4096
  // tokens, 32 + 8 heads of 128, pages of 16 607 us so, 488 from the lanes.  One or
  // two from the lanes: pages of 64 424 against 418, of 32 471 against 457.)
  __device__ __forceinline__ int64_t base_at(const CacheView& c, int32_t h, int u) const {
    int32_t p;
    if constexpr (GB == 1) {
      p = max(__builtin_amdgcn_readlane(lanes, lane0 + u), 0);
    } else {
      p = page[0];
#pragma unroll
      for (int n = 1; n < N; ++n) p = u / GB == n ? page[n] : p;
    }
    return (((int64_t)p * c.Hkv + h) << c.lp) * c.D;
  }
  __device__ __forceinline__ static int32_t slot(const CacheView& c, int32_t kb, int u) {
    return GB == 4 ? (kb & ((1 << c.lp) - 1)) + 16 * u : 16 * (u % GB);
  }
};

// A sequence's page numbers and scales, 64 pages at a time, one a lane.  The next
// 64 are loaded when the ones before them come into use, and the numbers of those
// after them, so that nothing waits for the two loads in a row that a page takes
// (as scalar loads, which share their counter with LDS reads, they held up every
// step for their latency).
template <int GB>
struct PageList {
  const int32_t* table;
  int32_t first;                       // page of lane 0
  int32_t page, ks, vs, page1, ks1, vs1, page2;
  __device__ __forceinline__ int32_t number(const CacheView& c, int32_t at, int lane) const {
    const int32_t p = table[min(at + lane, c.max_pages - 1)];
    return (uint32_t)p < (uint32_t)c.n_pages ? p : -1;
  }
  __device__ __forceinline__ static void scales(const CacheView& c, int32_t h, int32_t p,
                                                int32_t& k, int32_t& v) {
    const int64_t at = (int64_t)max(p, 0) * c.Hkv + h;
    k = c.k_scale[at];
    v = c.v_scale[at];
    k = p < 0 ? -1 : k;
  }
  __device__ __forceinline__ void numbers(const CacheView& c, const int32_t* t, int32_t kb, int lane) {
    table = t;
    first = kb >> c.lp;
    page = number(c, first, lane);
    page1 = number(c, first + 64, lane);
    page2 = number(c, first + 128, lane);
  }
  __device__ __forceinline__ void init(const CacheView& c, const int32_t* t, int32_t h, int32_t kb,
                                       int lane) {
    numbers(c, t, kb, lane);
    scales(c, h, page, ks, vs);
    scales(c, h, page1, ks1, vs1);
  }
  // init after numbers(kb0) with kb0 <= kb
  __device__ __forceinline__ void start(const CacheView& c, int32_t h, int32_t kb, int lane) {
    if ((kb >> c.lp) - first >= 64) numbers(c, table, kb, lane);
    scales(c, h, page, ks, vs);
    scales(c, h, page1, ks1, vs1);
  }
  // The pages at kb, which is not before the last one asked for and less than 64
  // pages past it, without their scales: those are scale()'s, to be asked for
  // before the next pages are, but after the loads from these have been issued.
  __device__ __forceinline__ Pages<GB> at(const CacheView& c, int32_t h, int32_t kb, int lane) {
    if ((kb >> c.lp) - first >= 64) {
      first += 64;
      page = page1;
      ks = ks1;
      vs = vs1;
      page1 = page2;
      scales(c, h, page1, ks1, vs1);
      page2 = number(c, first + 128, lane);
    }
    Pages<GB> r;
    const int32_t i = (kb >> c.lp) - first;
#pragma unroll
    for (int n = 0; n < Pages<GB>::N; ++n) {
      r.page[n] = max(__builtin_amdgcn_readlane(page, i + n), 0);
      r.ks[n] = r.vs[n] = 0;
    }
    if (GB == 1) {
      r.lanes = page;
      r.lane0 = i;
    }
    return r;
  }
  __device__ __forceinline__ void scale(const CacheView& c, int32_t kb, Pages<GB>& r) const {
    const int32_t i = (kb >> c.lp) - first;
#pragma unroll
    for (int n = 0; n < Pages<GB>::N; ++n) {
      r.ks[n] = __builtin_amdgcn_readlane(ks, i + n);
      r.vs[n] = __builtin_amdgcn_readlane(vs, i + n);
    }
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
    // (put together at once: word by word, heads of 256 spilled with one workgroup a
    // tile, 21.8 us for 64 sequences of up to 900 keys against 21.0, and kept one wave
    // a SIMD where the keys are split: 57.5 us for 8 of 16384 against 50.3)
    typedef int v2i __attribute__((ext_vector_type(2)));
    const v2i lo = *(const v2i*)(c.v + pg.base(c, h, 0) + g * 512 + lane * 8);
    const v2i hi = *(const v2i*)(c.v + pg.base(c, h, 2) + g * 512 + lane * 8);
    v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
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
// The same of m and c scaled by 2^4 (HI), where the host has shown that every
// multiplier stays below 2^27: the high word as it is.
template <bool HI>
__device__ __forceinline__ int32_t rescale(int32_t acc, int32_t m, int64_t c) {
  return HI ? (int32_t)(((int64_t)acc * m + c) >> 32) : rescale(acc, m, c);
}
// The multiplier of a row's products with the keys of a page.
__device__ __forceinline__ int32_t score_mult(int32_t A, int32_t ks) {
  // (the low word by a byte permute of both: from a 64-bit shift the compiler
  // would make the products below 64 x 64 bits wide)
  const int64_t p = (int64_t)A * ks + (1 << 15);
  return (int32_t)__builtin_amdgcn_perm((uint32_t)(p >> 32), (uint32_t)p, 0x05040302u);
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

// The sum of up to 2^17 products of low digits and values from its int32, which has
// wrapped where every one of 2^17 products is (-128)^2: 2^31 stands there as -2^31,
// which no sum is (the least is 2^17 * -128 * 127).
__device__ __forceinline__ int64_t low_sum(int32_t s) {
  return (int64_t)(int32_t)((uint32_t)s - 1) + 1;
}

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
  // |r| < 2^25; past +-clamp the result saturates (clamp_bound on the host), within
  // it the shifted product fits 32 bits
  __device__ __forceinline__ int32_t out(int64_t T, const CacheAttnArgs& a) const {
    const int32_t r = med3((int32_t)((T * (int64_t)F) >> sh), -a.out_clamp, a.out_clamp);
    const int64_t v = (int64_t)r * a.out_mult + ((int64_t)1 << (a.out_shift - 1));
    return med3((int32_t)(v >> a.out_shift), kQmin, kQmax);
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

// ---- many rows: a wave takes 16 NF rows of a (sequence, kv head) over all their
// keys twice.  The four waves of a workgroup share the keys and values of a step
// (64 keys) in LDS, where they come straight from memory, two steps side by side:
// the loads of a step are in flight during the products of the one before.
__device__ __forceinline__ void load_lds16(const int8_t* src, int8_t* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// 64 keys in LDS: keys [head_dim / 64][64][64 bytes], their 16-byte chunks
// swizzled as lds_chunk<4> has them (32-byte rows as they are), then the values as
// they lie in memory, page after page.
template <int D, int GB>
struct Step {
  static constexpr int CH = D >= 64 ? 4 : 2, BYTES = 64 * D;
  // byte of this lane's page base among the step's (uniform where it can be)
  template <int PER>
  __device__ static __forceinline__ int64_t page_base(const CacheView& c, const Pages<GB>& pg,
                                                      int32_t h, int q, int at) {
    // PER chunks a page: instruction q covers chunks 64 q .. 64 q + 63
    if constexpr (PER >= 64) {
      return pg.base_at(c, h, (q * 64 / PER) * GB);
    } else {
      static_assert(PER == 32, "half an instruction a page");
      const int64_t lo = pg.base_at(c, h, 2 * q * GB), hi = pg.base_at(c, h, (2 * q + 1) * GB);
      return at < 32 ? lo : hi;
    }
  }
  __device__ static __forceinline__ void keys(const CacheView& c, const Pages<GB>& pg, int32_t h,
                                              int32_t kb, int8_t* lds, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < (D / 16 + 3) / 4; ++q) {
      const int i = q * 4 + wave;  // chunks 64 i .. 64 i + 63 of [kc][64][CH]
      if (D < 64 && i >= D / 16) break;
      const int kc = i / CH, part = i % CH;  // 64 / CH rows of it
      const int row = part * (64 / CH) + lane / CH, ch = lane % CH;
      const int sw = CH == 4 ? ch ^ ((row & 4) >> 1) : ch;
      int64_t at;
      if constexpr (CH == 4) {
        at = pg.base_at(c, h, part) + (Pages<GB>::slot(c, kb, part) + (lane >> 2)) * D;
      } else if constexpr (GB == 1) {
        at = lane < 32 ? pg.base_at(c, h, 2 * part) : pg.base_at(c, h, 2 * part + 1);
        at += (row & 15) * D;
      } else {
        at = pg.base_at(c, h, 2 * part) + (Pages<GB>::slot(c, kb, 2 * part) + (lane >> 1)) * D;
      }
      load_lds16(c.k + at + kc * 64 + sw * 16, lds + i * 1024);
    }
  }
  __device__ static __forceinline__ void values(const CacheView& c, const Pages<GB>& pg, int32_t h,
                                                int32_t kb, int8_t* lds, int wave, int lane) {
    constexpr int PER = D * GB;  // 16-byte chunks a page
    const int32_t s0 = GB == 4 ? Pages<GB>::slot(c, kb, 0) * D : 0;
#pragma unroll
    for (int q = 0; q < (D / 16 + 3) / 4; ++q) {
      const int i = q * 4 + wave;
      if (D < 64 && i >= D / 16) break;
      load_lds16(c.v + page_base<PER>(c, pg, h, i, lane) + s0 + (i * 64 + lane) % PER * 16,
                 lds + i * 1024);
    }
  }
  __device__ static __forceinline__ v4i key(const int8_t* lds, int u, int kc, int lane) {
    const int r = u * 16 + (lane & 15), c = lane >> 4;
    if constexpr (CH == 4) return *(const v4i*)(lds + kc * 4096 + lds_chunk<4>(r, c));
    else return lane < 32 ? *(const v4i*)(lds + r * 32 + c * 16) : v4i{0, 0, 0, 0};
  }
  __device__ static __forceinline__ v4i value(const int8_t* lds, int g, int lane) {
    v4i v;
    if constexpr (GB == 4) {
      v = *(const v4i*)(lds + g * 1024 + lane * 16);
    } else if constexpr (GB == 2) {
      typedef int v2i __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const v2i x = *(const v2i*)(lds + i * (D * 32) + g * 512 + lane * 8);
        v[2 * i] = x[0];
        v[2 * i + 1] = x[1];
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *(const int32_t*)(lds + u * (D * 16) + g * 256 + lane * 4);
    }
    return v;
  }
};

// HI: rescale<true>.
template <int D, int GB, int NF, bool HI>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void cache_rows_kernel(CacheAttnArgs a, uint32_t tiles) {
  constexpr int CG = D / 16, KC = Keys<D>::KC, UP = HI ? 4 : 0;
  constexpr int64_t RND = kRnd << UP;
  typedef Step<D, GB> St;
  __shared__ __attribute__((aligned(1024))) int8_t even[2 * St::BYTES], odd[2 * St::BYTES];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t pair = blockIdx.x / tiles, tile = tiles - 1 - (blockIdx.x - pair * tiles);
  const int32_t s = (int32_t)(pair / (uint32_t)a.c.Hkv), h = (int32_t)(pair - (uint32_t)s * a.c.Hkv);
  const int32_t G = a.Hq / a.c.Hkv;
  const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;
  const Seq sq(a, s);
  const int32_t rows = sq.nq * G, w0 = (int32_t)tile * 64 * NF;
  if (w0 >= rows) return;
  // waves past the last row repeat it; their results are not stored
  const int32_t r0 = w0 + wave * 16 * NF;
  Rows<D, NF> R;
  R.load(a, sq, h, G, min(r0, rows - 1), rows, lane);
  const Span s0(a, sq, w0 / G), s1(a, sq, (min(w0 + 64 * NF, rows) - 1) / G);
  const int32_t kb0 = s0.lo & ~63, kend = s1.hi;
  auto full = [&](int32_t kb) { return kb >= R.all_lo && kb + 64 <= R.all_hi; };
  auto none = [&](int32_t kb) { return kb + 64 <= R.any_lo || kb >= R.any_hi; };
  const v4i zero = {0, 0, 0, 0};
  // body(kb, pages, tile) for every step; its tile (keys, then values) is complete,
  // and the other buffer free, at the barrier ahead of it
  auto steps = [&](auto with_values, auto body) {
    constexpr bool V = decltype(with_values)::value;
    PageList<GB> list;
    list.init(a.c, table, h, kb0, lane);
    Pages<GB> p0 = list.at(a.c, h, kb0, lane);
    auto load = [&](const Pages<GB>& pg, int32_t kb, int8_t* to) {
      St::keys(a.c, pg, h, kb, to, wave, lane);
      if (V) St::values(a.c, pg, h, kb, to + St::BYTES, wave, lane);
    };
    auto step = [&](int32_t kb, Pages<GB> pg, int8_t* tile, int8_t* other) {
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt 0
      lds_sync();
      list.scale(a.c, kb, pg);
      const Pages<GB> next = list.at(a.c, h, kb + 64, lane);
      if (kb + 64 < kend) load(next, kb + 64, other);
      if (!none(kb)) body(kb, pg, tile);
      return next;
    };
    lds_sync();  // (the last user of the buffers is done)
    if (kb0 < kend) load(p0, kb0, even);
    for (int32_t kb = kb0; kb < kend; kb += 128) {
      const Pages<GB> p1 = step(kb, p0, even, odd);
      if (kb + 64 >= kend) break;
      p0 = step(kb + 64, p1, odd, even);
    }
  };
  auto products = [&](const int8_t* buf, int u, v4i(&p)[NF]) {
#pragma unroll
    for (int f = 0; f < NF; ++f) p[f] = zero;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const v4i k = St::key(buf, u, kc, lane);
#pragma unroll
      for (int f = 0; f < NF; ++f)
        p[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k, R.q[f][kc], p[f], 0, 0, 0);
    }
  };

  // ---- maxima
  int32_t M[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) M[f] = kNone;
  steps(Flag<false>{}, [&](int32_t kb, const Pages<GB>& pg, const int8_t* keys) {
    if (full(kb) && pg.all()) {
      v4i top[NF];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v4i p[NF];
        products(keys, u, p);
        // (products of one scale are compared before they are rescaled)
#pragma unroll
        for (int f = 0; f < NF; ++f) {
#pragma unroll
          for (int r = 0; r < 4; ++r) top[f][r] = u % GB == 0 ? p[f][r] : max(top[f][r], p[f][r]);
          if (u % GB == GB - 1)
            M[f] = max(max(M[f], -32767),
                       rescale<HI>(max(max(top[f][0], top[f][1]), max(top[f][2], top[f][3])),
                                   score_mult(R.A[f], pg.ks[u / GB]) << UP, RND));
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v4i p[NF];
        products(keys, u, p);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const int32_t m = score_mult(R.A[f], pg.ks[u / GB]) << UP;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int32_t x = max(rescale<HI>(p[f][r], m, RND), -32767);
            M[f] = max(M[f], R.sees(f, kb + 16 * u + 4 * (lane >> 4) + r, pg.ks[u / GB]) ? x : kNone);
          }
        }
      }
    }
  });
  Ref ref[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    ref[f].init(over_lanes(M[f]));
    ref[f].c = ref[f].c * (1 << UP);
  }

  // ---- weights and sums
  v4i oh[CG][NF], ol[CG][NF];
  uint32_t L[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    L[f] = 0;
#pragma unroll
    for (int g = 0; g < CG; ++g) oh[g][f] = ol[g][f] = zero;
  }
  steps(Flag<true>{}, [&](int32_t kb, const Pages<GB>& pg, const int8_t* keys) {
    v4i ph[NF], pl[NF];
    auto weights = [&](auto checked) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v4i p[NF];
        products(keys, u, p);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const int32_t m = score_mult(R.A[f], pg.ks[u / GB]) << UP;
          uint32_t w[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            w[r] = weight(med3(rescale<HI>(p[f][r], m, ref[f].c), ref[f].cap, 0));
            if (decltype(checked)::value &&
                !R.sees(f, kb + 16 * u + 4 * (lane >> 4) + r, pg.ks[u / GB]))
              w[r] = 0;
          }
          L[f] += w[0] + w[1] + w[2] + w[3];
          const Digits d(w, (uint32_t)pg.vs[u / GB]);
          ph[f][u] = (int)d.hi;
          pl[f][u] = (int)d.lo;
        }
      }
    };
    if (full(kb) && pg.all()) weights(Flag<false>{});
    else weights(Flag<true>{});
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const v4i v = St::value(keys + St::BYTES, g, lane);
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        oh[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, ph[f], oh[g][f], 0, 0, 0);
        ol[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, pl[f], ol[g][f], 0, 0, 0);
      }
    }
  });
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
        v[r] = nm.out((int64_t)oh[g][f][r] * 256 + low_sum(ol[g][f][r]), a);
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
  int32_t tiles, rt, rpt, steps, nsplit, chunk;  // tiles a pair, rows a tile, keys a part
};

// The tile of a workgroup: its sequence, kv head and rows, and the keys that some
// of them see, end - base of them from a multiple of 64 on (0 where none is seen),
// in `parts` parts.
struct Few {
  int32_t s, h, G, r0, rows, base, end, parts;
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
    base = s0.lo & ~63;
    // (where none is seen, none is taken: no scores of keys from base to s0.lo are
    // written, and the one part of a tile goes on to its zeros)
    end = s1.hi > s0.lo ? s1.hi : base;
    parts = (end - base + sp.chunk - 1) / sp.chunk;
    return true;
  }
};

// Scores of the wave's steps (every NW-th from `wave` on) of keys c0 .. c1 - 1, to
// out(step, words); the row's maximum over them comes back.
template <int D, int GB, int NW, typename Out>
__device__ __forceinline__ int32_t few_scores(const CacheAttnArgs& a, const Rows<D, 1>& R,
                                              PageList<GB> list, int32_t h, int32_t c0,
                                              int32_t c1, int wave, int lane, Out out) {
  int32_t M = kNone;
  const int32_t kb0 = c0 + wave * 64;
  if (kb0 >= c1) return M;
  list.start(a.c, h, kb0, lane);
  Pages<GB> p0 = list.at(a.c, h, kb0, lane);
  Keys<D> k0;
  k0.load(a.c, p0, h, kb0, lane);
  // one step from pg and k, the next one's page and keys on their way to pn and kn
  auto step = [&](int32_t kb, Pages<GB>& pg, const Keys<D>& k, Pages<GB>& pn, Keys<D>& kn) {
    list.scale(a.c, kb, pg);
    // (past the last step too: any page number leads to a page)
    pn = list.at(a.c, h, kb + 64 * NW, lane);
    kn.load(a.c, pn, h, kb + 64 * NW, lane);
    v4i w[2];
    auto scores = [&](auto checked) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const v4i p = R.products(k, u, 0);
        const int32_t m = score_mult(R.A[0], pg.ks[u / GB]);
        int32_t x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = med3(rescale(p[r], m, kRnd), -32767, 32767);
          if (decltype(checked)::value)
            x[r] = R.sees(0, kb + 16 * u + 4 * (lane >> 4) + r, pg.ks[u / GB]) ? x[r] : kNone;
          M = max(M, x[r]);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
          w[u / 2][(u % 2) * 2 + r] = (int)__builtin_amdgcn_perm((uint32_t)x[2 * r + 1],
                                                                 (uint32_t)x[2 * r], 0x05040100u);
      }
    };
    if (kb >= R.all_lo && kb + 64 <= R.all_hi && pg.all()) scores(Flag<false>{});
    else scores(Flag<true>{});
    out(kb >> 6, w);
  };
  Pages<GB> p1;
  Keys<D> k1;
  for (int32_t kb = kb0; kb < c1; kb += 128 * NW) {
    step(kb, p0, k0, p1, k1);
    if (kb + 64 * NW >= c1) break;
    step(kb + 64 * NW, p1, k1, p0, k0);
  }
  return M;
}

// Weights and sums of the same steps, the scores from in(step); the reference
// from top(), which may wait for the other waves, once the first values are on
// their way.
template <int D, int GB, int NW, typename Top, typename In>
__device__ __forceinline__ uint32_t few_values(const CacheAttnArgs& a, PageList<GB> list, int32_t h,
                                               int32_t c0, int32_t c1, int wave, int lane, Top top,
                                               In in, v4i (&oh)[D / 16], v4i (&ol)[D / 16]) {
  // values are loaded a step ahead where registers are left for a second set (with
  // 256 channels that spilled: 700 keys 26 us so, 16 now; 8 x 16384 keys 29 and 22)
  constexpr bool AHEAD = D < 256;
  constexpr int CG = D / 16;
  uint32_t L = 0;
  const v4i zero = {0, 0, 0, 0};
#pragma unroll
  for (int g = 0; g < CG; ++g) oh[g] = ol[g] = zero;
  const int32_t kb0 = c0 + wave * 64;
  auto load = [&](const Pages<GB>& pg, int32_t kb, v4i(&v)[CG]) {
#pragma unroll
    for (int g = 0; g < CG; ++g) v[g] = load_values<D, GB>(a.c, pg, h, kb, g, lane);
  };
  Pages<GB> p0;
  v4i v0[CG];
  if (kb0 < c1) {
    list.start(a.c, h, kb0, lane);
    p0 = list.at(a.c, h, kb0, lane);
    load(p0, kb0, v0);
  }
  // (a wave's own scores: no other wave's are read)
  v4i x0[2];
  if (kb0 < c1) in(kb0 >> 6, x0);
  const Ref ref = top();
  auto step = [&](int32_t kb, Pages<GB>& pg, v4i(&v)[CG], const v4i(&x)[2], Pages<GB>& pn,
                  v4i(&vn)[CG], v4i(&xn)[2]) {
    if (kb + 64 * NW < c1) in((kb >> 6) + NW, xn);
    list.scale(a.c, kb, pg);
    if (!AHEAD && kb != kb0) load(pg, kb, v);
    pn = list.at(a.c, h, kb + 64 * NW, lane);
    if (AHEAD) load(pn, kb + 64 * NW, vn);
    v4i ph, pl;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int32_t two = x[u / 2][(u % 2) * 2 + r / 2];
        const int32_t sc = r % 2 ? two >> 16 : (int16_t)two;
        // (made for all of them: a choice between 0 and what inline asm has part in
        // becomes a branch, 16 a step: 700 keys of 64 channels 8.1 us so, 7.0 now)
        const uint32_t all = weight(med3(sc - ref.m, ref.cap, 0));
        w[r] = sc == kNone ? 0 : all;
      }
      L += w[0] + w[1] + w[2] + w[3];
      const Digits d(w, (uint32_t)pg.vs[u / GB]);
      ph[u] = (int)d.hi;
      pl[u] = (int)d.lo;
    }
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      oh[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[g], ph, oh[g], 0, 0, 0);
      ol[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[g], pl, ol[g], 0, 0, 0);
    }
  };
  if constexpr (AHEAD) {
    Pages<GB> p1;
    v4i v1[CG], x1[2];
    for (int32_t kb = kb0; kb < c1; kb += 128 * NW) {
      step(kb, p0, v0, x0, p1, v1, x1);
      if (kb + 64 * NW >= c1) break;
      step(kb + 64 * NW, p1, v1, x1, p0, v0, x0);
    }
  } else {
#pragma unroll 1
    for (int32_t kb = kb0; kb < c1; kb += 64 * NW) {
      Pages<GB> p1;
      v4i x1[2];
      step(kb, p0, v0, x0, p1, v0, x1);
      p0 = p1;
      x0[0] = x1[0];
      x0[1] = x1[1];
    }
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

  // A tile's output.
  template <typename Few>
  __device__ __forceinline__ void write(const CacheAttnArgs& a, const Few& t, int32_t first,
                                        int32_t rows) const {
    for (int i = threadIdx.x; i < D / 16 * 64; i += 64 * NW) {
      const int ln = i & 63, g = i >> 6, row = ln & 15;
      if (row >= rows) continue;
      Norm nm;
      nm.init(L[row]);
      int32_t v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = nm.out(T(i * 4 + k), a);
      const int32_t r = t.r0 + row, q = r / t.G;
      *(uint32_t*)(a.out + ((int64_t)(first + q) * a.Hq + t.h * t.G + r - q * t.G) * D + g * 16 +
                   (ln >> 4) * 4) = pack4(v[0], v[1], v[2], v[3]);
    }
  }
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
  PageList<GB> list;
  list.numbers(a.c, a.c.table + (int64_t)t.s * a.c.max_pages, wave * 64, lane);
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq)) return;
  Rows<D, 1> R;
  R.load(a, sq, t.h, t.G, t.r0, t.rows, lane);
  const int32_t n = min(16, t.rows - t.r0);
  int16_t* scores = (int16_t*)dyn + (lane >> 4) * 16 + (lane & 15) * 64;
  const int32_t stride = sp.rpt * 64, s0 = t.base >> 6;
  sums.clear();
  const int32_t M = over_lanes(few_scores<D, GB, NW>(
      a, R, list, t.h, t.base, t.end, wave, lane, [&](int32_t step, const v4i(&w)[2]) {
        if ((lane & 15) >= n) return;
        v4i* p = (v4i*)(scores + (step - s0) * stride);
        p[0] = w[0];
        p[1] = w[1];
      }));
  if (lane < 16) top[wave][lane] = M;
  v4i oh[D / 16], ol[D / 16];
  const int32_t back = max((lane & 15) - (n - 1), 0) * 64;  // rows past the last repeat it
  const uint32_t L = few_values<D, GB, NW>(
      a, list, t.h, t.base, t.end, wave, lane,
      [&] {
        lds_sync();
        int32_t m = kNone;
#pragma unroll
        for (int w = 0; w < NW; ++w) m = max(m, top[w][lane & 15]);
        Ref ref;
        ref.init(m);
        return ref;
      },
      [&](int32_t step, v4i(&x)[2]) {
        const v4i* p = (const v4i*)(scores + (step - s0) * stride - back);
        x[0] = p[0];
        x[1] = p[1];
      }, oh, ol);
  sums.add(L, oh, ol, n, lane);
  lds_sync();
  sums.write(a, t, sq.first, n);
}

// Several workgroups a tile, in launches of their own: scores and maxima, sums,
// and, where a tile has several parts, the output.
template <int D, int GB>
__global__ __launch_bounds__(256) void split_scores_kernel(CacheAttnArgs a, Split sp) {
  __shared__ int32_t top[4][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (a part's tiles side by side: later parts are shorter or empty, and with a
  // tile's parts side by side some XCDs had only those: the sums of 32
  // sequences of up to 8192 keys 5% slower)
  const uint32_t part_u = blockIdx.x / (uint32_t)sp.tiles, tile = blockIdx.x - part_u * (uint32_t)sp.tiles;
  const int32_t part = (int32_t)part_u;
  Few t(a, sp, tile);
  PageList<GB> list;
  list.numbers(a.c, a.c.table + (int64_t)t.s * a.c.max_pages, part * sp.chunk + wave * 64, lane);
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq) || part >= t.parts) return;
  Rows<D, 1> R;
  R.load(a, sq, t.h, t.G, t.r0, t.rows, lane);
  const int32_t n = min(16, t.rows - t.r0);
  const int32_t c0 = t.base + part * sp.chunk, c1 = min(c0 + sp.chunk, t.end);
  int16_t* scores = sp.scores + ((int64_t)tile * sp.steps - (t.base >> 6)) * sp.rpt * 64 +
                    (lane >> 4) * 16 + (lane & 15) * 64;
  const int32_t M = over_lanes(few_scores<D, GB, 4>(
      a, R, list, t.h, c0, c1, wave, lane, [&](int32_t step, const v4i(&w)[2]) {
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
  __shared__ int32_t top[4][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (numbered as in the scores)
  const uint32_t part_u = blockIdx.x / (uint32_t)sp.tiles, tile = blockIdx.x - part_u * (uint32_t)sp.tiles;
  const int32_t part = (int32_t)part_u;
  Few t(a, sp, tile);
  PageList<GB> list;
  list.numbers(a.c, a.c.table + (int64_t)t.s * a.c.max_pages, part * sp.chunk + wave * 64, lane);
  const Seq sq(a, t.s);
  if (!t.bounds(a, sp, sq)) return;
  const int32_t n = min(16, t.rows - t.r0);
  // (without a join the only part writes the output, zeros where no key is seen)
  if (part >= t.parts && sp.nsplit > 1) return;
  const int32_t c0 = t.base + part * sp.chunk, c1 = min(c0 + sp.chunk, t.end);
  sums.clear();
  const int16_t* scores = sp.scores + ((int64_t)tile * sp.steps - (t.base >> 6)) * sp.rpt * 64 +
                          (lane >> 4) * 16 + min(lane & 15, n - 1) * 64;
  v4i oh[D / 16], ol[D / 16];
  const uint32_t L = few_values<D, GB, 4>(
      a, list, t.h, c0, c1, wave, lane,
      [&] {
        // the parts' maxima, 16 side by side
        const int32_t* all = sp.top + (int64_t)tile * sp.nsplit * 16 + (lane & 15);
        int32_t m = kNone;
#pragma unroll 4
        for (int32_t i = wave * 4 + (lane >> 4); i < t.parts; i += 16)
          m = max(m, all[i * 16]);
        m = over_lanes(m);
        if (lane < 16) top[wave][lane] = m;
        lds_sync();
#pragma unroll
        for (int w = 0; w < 4; ++w) m = max(m, top[w][lane & 15]);
        Ref ref;
        ref.init(m);
        return ref;
      },
      [&](int32_t step, v4i(&x)[2]) {
        const v4i* p = (const v4i*)(scores + (int64_t)step * sp.rpt * 64);
        x[0] = p[0];
        x[1] = p[1];
      }, oh, ol);
  sums.add(L, oh, ol, n, lane);
  lds_sync();
  if (sp.nsplit == 1) {
    sums.write(a, t, sq.first, n);
    return;
  }
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
  for (int32_t i = p0; i < t.parts; i += PP) {
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
    v[k] = nm.out(x, a);
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
  int64_t tiles;   // of 16 rows
  int64_t rows, shared;  // of a kv head; workgroups of ROWS
  size_t bytes;    // of the workspace
};
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

Plan plan(const CacheAttnArgs& a) {
  Plan p = {};
  const int64_t G = a.Hq / a.c.Hkv, rows = a.max_q * G, pairs = (int64_t)a.seqs * a.c.Hkv;
  p.sp.rt = (int32_t)((rows + 15) / 16);
  p.sp.rpt = (int32_t)(rows < 16 ? rows : 16);
  // keys that a tile's rows (at most 16 queries) can see
  const int64_t seen = a.window && (int64_t)a.window + 16 < a.max_len ? a.window + 16 : a.max_len;
  p.sp.steps = (int32_t)((seen + 63) / 64) + (seen < a.max_len);
  p.tiles = pairs * p.sp.rt;
  p.sp.tiles = (int32_t)p.tiles;
  p.sp.nsplit = 1;
  p.sp.chunk = p.sp.steps * 64 + 64;
  if (p.tiles == 0 || p.sp.steps == 0) {
    p.way = FEW;
    return p;
  }
  // Many rows, and enough of them to fill the CUs: the kernel that shares keys
  // among the rows of a workgroup (128, or 64 of 256 channels).  16 heads of 600
  // queries over 4696 keys each are 80 workgroups: 110 us so, 59 us split.
  p.rows = rows;
  p.shared = pairs * ((rows + (a.c.D >= 256 ? 63 : 127)) / (a.c.D >= 256 ? 64 : 128));
  if (rows > 64 && p.shared >= 192 && a.max_len <= 131072) {
    p.way = ROWS;
    return p;
  }
  const size_t lds = (size_t)p.sp.steps * p.sp.rpt * 128;
  if (seen <= 1024 && lds <= 32768) {
    p.way = FEW;
    return p;
  }
  p.way = SPLIT;
  // Parts enough for two workgroups a CU, of at least 512 keys, if every sequence had
  // max_len of them (what they have is on the device).  (One sequence of 131072 keys
  // and 8 kv heads in 512, 1024 and 2048 parts: 30, 32 and 36 us for the scores, 29,
  // 34 and 42 for the sums: a part costs its start.  Of ragged sequences the longest
  // sets the time: 32 of 2227 to 8192 keys, 5148 on average, take 1.6 times their
  // bytes' time, and finer parts were not measured on them.)
  int64_t chunk = (seen * p.tiles + 511) / 512;
  chunk = (chunk + 255) / 256 * 256;
  if (chunk < 512) chunk = 512;
  if (chunk > 32768) chunk = 32768;
  p.sp.chunk = (int32_t)chunk;
  p.sp.nsplit = (int32_t)((p.sp.steps * 64 + chunk - 1) / chunk);
  const int64_t parts = p.tiles * p.sp.nsplit;
  p.bytes = align256((size_t)p.tiles * p.sp.steps * p.sp.rpt * 128) + align256((size_t)parts * 64);
  if (p.sp.nsplit > 1)
    p.bytes += align256((size_t)parts * p.sp.rpt * a.c.D * 8) + align256((size_t)parts * 128);
  return p;
}

template <int D, int GB>
hipError_t launch_pages(const CacheAttnArgs& a, void* ws, hipStream_t s) {
  Plan p = plan(a);
  if (p.tiles == 0) return hipSuccess;
  if (p.way == ROWS) {
    constexpr int NF = D >= 256 ? 1 : 2;
    const uint32_t tiles = (uint32_t)((p.rows + 64 * NF - 1) / (64 * NF));
    const int64_t total = p.shared;
    // the largest multiplier that scales within their bounds can make
    const int64_t A = (33026 * (int64_t)a.score_mult + ((int64_t)1 << (a.score_t - 1))) >> a.score_t;
    if ((A * 37154 + (1 << 15)) >> 16 < (1 << 27))
      hipLaunchKernelGGL((cache_rows_kernel<D, GB, NF, true>), dim3((unsigned)total), dim3(256), 0, s,
                         a, tiles);
    else
      hipLaunchKernelGGL((cache_rows_kernel<D, GB, NF, false>), dim3((unsigned)total), dim3(256), 0,
                         s, a, tiles);
    return hipGetLastError();
  }
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
  if ((e = hipGetLastError()) != hipSuccess || p.sp.nsplit == 1) return e;
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

// (every grid below 2^32 threads)
bool cache_attention_fits(const CacheAttnArgs& a) {
  const Plan p = plan(a);
  if (p.way == ROWS) return p.shared < ((int64_t)1 << 24);
  return p.tiles * p.sp.nsplit < ((int64_t)1 << 23) && p.tiles * 16 < ((int64_t)1 << 24);
}

hipError_t launch_cache_attention(const CacheAttnArgs& args, void* ws, hipStream_t s) {
  CacheAttnArgs a = args;
  // beyond |r| = L the output saturates: |r m| >= 129 2^s (r stays below 2^25)
  const int64_t am = a.out_mult < 0 ? -(int64_t)a.out_mult : (int64_t)a.out_mult;
  const int64_t L = am && a.out_shift <= 54 ? 129 * ((int64_t)1 << a.out_shift) / am + 1 : 1 << 30;
  a.out_clamp = (int32_t)(L < (1 << 30) ? L : 1 << 30);
  switch (a.c.D) {
    case 32: return launch_dim<32>(a, ws, s);
    case 64: return launch_dim<64>(a, ws, s);
    case 128: return launch_dim<128>(a, ws, s);
    default: return launch_dim<256>(a, ws, s);
  }
}

}  // namespace ilw
