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
// or two or four.  GB: 16-key blocks of a page among them.
template <int GB>
struct Pages {
  static constexpr int N = 4 / GB;
  int32_t page[N], ks[N], vs[N];
  bool ok[N];
  __device__ __forceinline__ void load(const CacheView& c, const int32_t* table, int32_t h,
                                       int32_t kb) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int32_t p = table[min((kb >> c.lp) + i, c.max_pages - 1)];
      ok[i] = (uint32_t)p < (uint32_t)c.n_pages;
      page[i] = ok[i] ? p : 0;
      const int64_t at = (int64_t)page[i] * c.Hkv + h;
      ks[i] = c.k_scale[at];
      vs[i] = c.v_scale[at];
    }
  }
  __device__ __forceinline__ bool all() const {
    bool r = true;
#pragma unroll
    for (int i = 0; i < N; ++i) r = r && ok[i];
    return r;
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

// One wave for 16 NF rows of a (sequence, kv head), over all their keys twice.
template <int D, int GB, int NF>
__global__ __launch_bounds__(256) void cache_rows_kernel(CacheAttnArgs a, uint32_t tiles) {
  constexpr int KC = Keys<D>::KC, CG = D / 16;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t pair = blockIdx.x / tiles, tile = tiles - 1 - (blockIdx.x - pair * tiles);
  const int32_t s = (int32_t)(pair / (uint32_t)a.c.Hkv), h = (int32_t)(pair - (uint32_t)s * a.c.Hkv);
  const int32_t G = a.Hq / a.c.Hkv;
  const Seq sq(a, s);
  const int32_t rows = sq.nq * G, r0 = ((int32_t)tile * 4 + wave) * 16 * NF;
  if (r0 >= rows) return;
  const int32_t* table = a.c.table + (int64_t)s * a.c.max_pages;

  // this lane's rows (the columns of the products); rows past the last repeat it
  int32_t A[NF], lo[NF], hi[NF];
  v4i qf[NF][KC];
  int64_t at[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    const int32_t r = min(r0 + f * 16 + (lane & 15), rows - 1), i = r / G, g = r - i * G;
    const Span sp(a, sq, i);
    lo[f] = sp.lo;
    hi[f] = sp.hi;
    at[f] = (int64_t)(sq.first + i) * a.Hq + h * G + g;
    A[f] = (int32_t)(((int64_t)a.q_scale[at[f]] * a.score_mult + ((int64_t)1 << (a.score_t - 1))) >>
                     a.score_t);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
      qf[f][kc] = D >= 64 || lane < 32
                      ? *(const v4i*)(a.q + at[f] * D + kc * 64 + (lane >> 4) * 16)
                      : v4i{0, 0, 0, 0};
  }
  // the wave's keys: every row's span lies in [first.lo, last.hi), and keys in
  // [last.lo, first.hi) are seen by every row
  const Span s0(a, sq, r0 / G), s1(a, sq, (min(r0 + 16 * NF, rows) - 1) / G);
  const int32_t kb0 = s0.lo & ~63, kend = s1.hi;
  auto full = [&](int32_t kb) { return kb >= s1.lo && kb + 64 <= s0.hi; };
  const v4i zero = {0, 0, 0, 0};
  auto products = [&](const Keys<D>& k, int u, int f) {
    v4i p = zero;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
      p = __builtin_amdgcn_mfma_i32_16x16x64_i8(k.f[u][kc], qf[f][kc], p, 0, 0, 0);
    return p;
  };

  int32_t M[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) M[f] = kNone;
  for (int32_t kb = kb0; kb < kend; kb += 64) {
    Pages<GB> pg;
    pg.load(a.c, table, h, kb);
    Keys<D> k;
    k.load(a.c, pg, h, kb, lane);
    const bool fast = full(kb) && pg.all();
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const v4i p = products(k, u, f);
        const int32_t m = score_mult(A[f], pg.ks[u / GB]);
        if (fast) {
          M[f] = max(max(M[f], -32767), rescale(max(max(p[0], p[1]), max(p[2], p[3])), m, kRnd));
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int32_t key = kb + 16 * u + 4 * (lane >> 4) + r;
            const bool see = key >= lo[f] && key < hi[f] && pg.ok[u / GB];
            M[f] = max(M[f], see ? max(rescale(p[r], m, kRnd), -32767) : kNone);
          }
        }
      }
  }
  int64_t c[NF];
  int32_t cap[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    M[f] = max(M[f], __shfl_xor(M[f], 16, 64));
    M[f] = max(M[f], __shfl_xor(M[f], 32, 64));
    M[f] = M[f] == kNone ? kNone : med3(M[f], -32767, 32767);
    c[f] = kRnd - (int64_t)M[f] * (1 << 28);
    // scores stop at -32767
    cap[f] = -min(kFar, M[f] + 32767);
  }
  v4i oh[CG][NF], ol[CG][NF];
  uint32_t L[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    L[f] = 0;
#pragma unroll
    for (int g = 0; g < CG; ++g) oh[g][f] = ol[g][f] = zero;
  }
  for (int32_t kb = kb0; kb < kend; kb += 64) {
    Pages<GB> pg;
    pg.load(a.c, table, h, kb);
    Keys<D> k;
    k.load(a.c, pg, h, kb, lane);
    const bool fast = full(kb) && pg.all();
    v4i ph[NF], pl[NF];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const v4i p = products(k, u, f);
        const int32_t m = score_mult(A[f], pg.ks[u / GB]);
        uint32_t d[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          uint32_t w = weight(med3(rescale(p[r], m, c[f]), cap[f], 0));
          if (!fast) {
            const int32_t key = kb + 16 * u + 4 * (lane >> 4) + r;
            w = key >= lo[f] && key < hi[f] && pg.ok[u / GB] ? w : 0;
          }
          L[f] += w;
          d[r] = __umul24(w, (uint32_t)pg.vs[u / GB]) + kDigits;
        }
        const uint32_t d01 = __builtin_amdgcn_perm(d[1], d[0], 0x07030602u);
        const uint32_t d23 = __builtin_amdgcn_perm(d[3], d[2], 0x07030602u);
        pl[f][u] = (int)(__builtin_amdgcn_perm(d23, d01, 0x05040100u) ^ 0x80808080u);
        ph[f][u] = (int)__builtin_amdgcn_perm(d23, d01, 0x07060302u);
      }
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const v4i v = load_values<D, GB>(a.c, pg, h, kb, g, lane);
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        oh[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, ph[f], oh[g][f], 0, 0, 0);
        ol[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, pl[f], ol[g][f], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    uint64_t l = L[f];
    l += (uint64_t)(uint32_t)__shfl_xor((int)L[f], 16, 64);
    const uint32_t l0 = __shfl_xor((int)(uint32_t)l, 32, 64), l1 = __shfl_xor((int)(l >> 32), 32, 64);
    l += ((uint64_t)l1 << 32) | l0;
    Norm nm;
    nm.init(l);
    if (r0 + f * 16 + (lane & 15) >= rows) continue;
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      int32_t v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[r] = nm.out((int64_t)oh[g][f][r] * 256 + ol[g][f][r], a.out_mult, a.out_shift);
      *(uint32_t*)(a.out + at[f] * D + g * 16 + (lane >> 4) * 4) = pack4(v[0], v[1], v[2], v[3]);
    }
  }
}

template <int D, int GB>
hipError_t launch_rows(const CacheAttnArgs& a, hipStream_t s) {
  constexpr int NF = D >= 256 ? 1 : 2;
  const int64_t rows = (int64_t)a.max_q * (a.Hq / a.c.Hkv);
  const uint32_t tiles = (uint32_t)((rows + 64 * NF - 1) / (64 * NF));
  const int64_t total = (int64_t)tiles * a.seqs * a.c.Hkv;
  if (total >= ((int64_t)1 << 24)) return hipErrorInvalidValue;  // under 2^32 threads
  hipLaunchKernelGGL((cache_rows_kernel<D, GB, NF>), dim3((unsigned)total), dim3(256), 0, s, a, tiles);
  return hipGetLastError();
}

template <int D>
hipError_t launch_dim(const CacheAttnArgs& a, hipStream_t s) {
  return a.c.lp >= 6 ? launch_rows<D, 4>(a, s)
                     : a.c.lp == 5 ? launch_rows<D, 2>(a, s) : launch_rows<D, 1>(a, s);
}

}  // namespace

size_t cache_attention_workspace(const CacheAttnArgs&) { return 0; }

hipError_t launch_cache_attention(const CacheAttnArgs& a, void*, hipStream_t s) {
  switch (a.c.D) {
    case 32: return launch_dim<32>(a, s);
    case 64: return launch_dim<64>(a, s);
    case 128: return launch_dim<128>(a, s);
    default: return launch_dim<256>(a, s);
  }
}

}  // namespace ilw
