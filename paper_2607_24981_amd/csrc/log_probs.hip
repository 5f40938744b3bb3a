// log_probs.hip -- log probabilities of given tokens, the entropy and the best
// alternatives of rows of int16 vocabulary scores (1/64 octave; -32768: not to be had).
//
// With a = max s - s and w = 2^(30 - a/64) (a table of 64 values, shifted), L = sum w
// and B = sum w a are exact in 64 bits (w <= 2^30, a < 31 * 64, 2^20 scores), so no
// order of the sums and no split of a row changes them; log2 p = (s - max s)/64 -
// log2(L / 2^30) and the entropy is log2(L / 2^30) + B / (64 L), both in 2^-16.  The
// maximum has to be known first: a running maximum would round the weights anew at
// each step.  So a row (or a part of one) stays in the registers of a workgroup, 8
// scores to a 16-byte unit, and is read once.
//
// Bound: 200 rows of 100003 scores take 16.8 us without alternatives, 10.4 of them to
// read (a workgroup a CU) and the rest for the weights and their sums, about ten vector
// instructions a score that cannot begin before the last score is there.  (A table of
// all 1985 weights saves the shifts and costs as much in LDS conflicts.)
//
// The best n: each of 256 groups of lanes has its largest score; the n-th largest of
// these is at most the n-th largest of all, and what is not below it goes to a list in
// LDS (about n + n^2/512 scores where the largest lie anywhere).  Each entry's rank is
// the number of larger keys (score, then lower index).  Where the list gets too long (ties),
// the n-th largest score itself is found by halving the range of scores, over the
// registers.
//
// A row with many scores and few rows beside it is cut in parts: their maxima and
// best n in one launch, their sums in a second, a third joins them.  (Joined by the
// last workgroup of a row instead, with a fence and a count in each: 60 rows of 200003
// scores 49 us.)
#include "step_internal.h"

namespace ilw {
namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2s __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Two scores of a word (by value: bit_cast of a vector's element takes its first).
__device__ __forceinline__ s16x2 pair(uint32_t w) { return __builtin_bit_cast(s16x2, w); }

constexpr uint32_t NONE2 = 0x80008000u;  // two scores that are not to be had
constexpr int32_t FAR = 31 * 64;         // weights from here on are 0
constexpr int GROUPS = 256;
constexpr int CAP = 1024;                // entries of the list
constexpr int MAXN = 64;
constexpr int MAXP = 64;  // parts of a row

// Parts' results between the launches.
struct PartView {
  int32_t* top;                 // [rows * P] largest score
  unsigned long long* sums;     // [rows * P][2] L, B
  unsigned long long* keys;     // [rows * P][n] the best, sorted
};

__device__ __forceinline__ unsigned long long key_of(int32_t s, int32_t v) {
  return ((unsigned long long)(uint32_t)(s + 32768) << 32) | (uint32_t)~v;
}
__device__ __forceinline__ int32_t key_score(unsigned long long k) { return (int32_t)(k >> 32) - 32768; }
__device__ __forceinline__ int32_t key_index(unsigned long long k) { return (int32_t)~(uint32_t)k; }

// log2(L / 2^30) in 2^-16, L >= 2^30: its 31 leading bits squared 16 times.
__device__ __forceinline__ int32_t log2_q16(uint64_t L) {
  const int32_t n = bit_length(L);
  uint64_t y = L >> (n - 31);
  int32_t frac = 0;
  for (int i = 0; i < 16; ++i) {
    y = (y * y) >> 30;
    const uint32_t up = (uint32_t)(y >> 31);
    y >>= up;
    frac = 2 * frac + (int32_t)up;
  }
  return ((n - 31) << 16) + frac;
}
__device__ __forceinline__ int32_t entropy_q16(int32_t lg, uint64_t L, uint64_t B) {
  const uint64_t q = B / L;
  return lg + (int32_t)((q << 10) + (((B - q * L) << 10) / L));
}
__device__ __forceinline__ int32_t log_prob(int32_t s, int32_t top, int32_t lg) {
  return s == kNoScore ? kNoLogProb : (s - top) * 1024 - lg;
}

__device__ __forceinline__ uint32_t at_byte(const uint32_t* table, uint32_t offset) {
  return *(const uint32_t*)((const int8_t*)table + offset);
}
// What a row's results are written from.
__device__ __forceinline__ void write_given(const LogProbArgs& a, int64_t row, int32_t top,
                                            int32_t lg, int tid, int nt) {
  for (int32_t i = tid; i < a.n_given; i += nt) {
    const int32_t v = a.given[row * a.n_given + i];
    const int32_t s = (uint32_t)v < (uint32_t)a.V ? a.logits[row * a.ld + v] : kNoScore;
    a.given_lp[row * a.n_given + i] = log_prob(s, top, lg);
  }
}

// The scores lo .. hi - 1 of the 8 from i on.
__device__ __forceinline__ u32x4 part_of_unit(const int16_t* base, int32_t i, int32_t lo, int32_t hi) {
  uint64_t w[2];
  for (int h = 0; h < 2; ++h) {
    w[h] = ((uint64_t)NONE2 << 32) | NONE2;
#pragma unroll 1
    for (int32_t v = max(i + 4 * h, lo); v < min(i + 4 * h + 4, hi); ++v) {
      const int32_t sh = 16 * (v - i - 4 * h);
      w[h] ^= (uint64_t)(uint16_t)(base[v] ^ kNoScore) << sh;
    }
  }
  return u32x4{(uint32_t)w[0], (uint32_t)(w[0] >> 32), (uint32_t)w[1], (uint32_t)(w[1] >> 32)};
}

enum { ALL = 0, BEST = 1, SUMS = 2 };

template <int NT, int U, int MODE>
__global__ __launch_bounds__(NT) void log_probs_kernel(LogProbArgs a, PartView ws, int32_t P) {
  constexpr int WAVES = NT / 64, GL = NT / GROUPS;  // lanes of a group
  __shared__ uint32_t table[64];
  __shared__ int32_t wave_top[WAVES], group_top[GROUPS];
  __shared__ unsigned long long wave_sum[WAVES][2];
  __shared__ unsigned long long list[MODE == SUMS ? 1 : CAP];
  __shared__ int32_t count, bound, lg_shared, tally[2][WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x / (uint32_t)P;
  const int32_t part = (int32_t)(blockIdx.x - (uint32_t)row * (uint32_t)P);
  const int32_t v0 = (int32_t)((int64_t)a.V * part / P), v1 = (int32_t)((int64_t)a.V * (part + 1) / P);
  const int32_t n_top = a.n_top;

  // units of 8 scores on 16-byte borders; off: scores before v0 in the first one
  const int16_t* first = a.logits + row * a.ld + v0;
  const int32_t off = (int32_t)(((uintptr_t)first & 15) >> 1), len = v1 - v0;
  const int16_t* base = first - off;
  u32x4 s[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t i = (uint32_t)(tid + k * NT) * 8;
    s[k] = u32x4{NONE2, NONE2, NONE2, NONE2};
    if (i >= (uint32_t)off && i + 8 <= (uint32_t)(off + len)) s[k] = *(const u32x4*)(base + i);
  }
  // the units that the row's part begins and ends in
  if (off > 0 && tid == 0) s[0] = part_of_unit(base, 0, off, off + len);
  const int32_t last = (off + len) >> 3;
  if (((off + len) & 7) && tid == last % NT) {
    const u32x4 w = part_of_unit(base, last * 8, off, off + len);
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (last / NT == k) s[k] = w;
  }
  load_exp2(table);
  if (tid == 0) count = 0;

  int32_t top;
  if (MODE == SUMS) {
    top = wave_max_i32(lane < P ? ws.top[row * P + lane] : kNoScore);  // (at most 64 parts)
    __syncthreads();
  } else {
    s16x2 m = {kNoScore, kNoScore};
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, pair(s[k][j]));
    int32_t g = max((int32_t)m.x, (int32_t)m.y);
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) g = max(g, __shfl_xor(g, o, 64));
    if (tid % GL == 0) group_top[tid / GL] = g;
#pragma unroll
    for (int o = GL; o < 64; o <<= 1) g = max(g, __shfl_xor(g, o, 64));
    if (lane == 0) wave_top[wave] = g;
    __syncthreads();
    top = wave_top[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = max(top, wave_top[i]);
  }

  if (MODE != BEST) {
    uint64_t L = 0, B = 0;
    const uint32_t top2 = ((uint32_t)top & 0xffffu) * 0x10001u;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      __builtin_amdgcn_sched_barrier(0);  // (a unit's weights at a time: more would spill)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u16x2s d = __builtin_bit_cast(u16x2s, top2) - __builtin_bit_cast(u16x2s, pair(s[k][j]));
        d = __builtin_elementwise_min(d, u16x2s{FAR, FAR});
        const uint32_t a = __builtin_bit_cast(uint32_t, d),
                       a4 = __builtin_bit_cast(uint32_t, d << u16x2s{2, 2});
        const uint32_t w0 = at_byte(table, a4 & 0xfcu) >> ((a >> 6) & 31),
                       w1 = at_byte(table, (a4 >> 16) & 0xffu) >> (a >> 22);
        L += w0 + w1;  // at most 2^31
        B += (uint64_t)w0 * (a & 0xffffu);
        B += (uint64_t)w1 * (a >> 16);
      }
    }
    if (top < kNoScore + FAR) {
      // -32768 itself was given a weight, that of top + 32768
      uint32_t none = 0;
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          none += ((s[k][j] & 0xffffu) == 0x8000u) + ((s[k][j] >> 16) == 0x8000u);
      const uint32_t d = (uint32_t)(top - kNoScore), w = exp2_q30(table, d);
      L -= (uint64_t)none * w;
      B -= (uint64_t)none * w * d;
    }
    L = wave_sum_u64(L);
    B = wave_sum_u64(B);
    if (lane == 0) wave_sum[wave][0] = L, wave_sum[wave][1] = B;
  }

  if (MODE != SUMS && n_top > 0) {
    if (wave == 0) {  // the n-th largest of the groups' maxima, by halving
      int32_t g[GROUPS / 64];
#pragma unroll
      for (int i = 0; i < GROUPS / 64; ++i) g[i] = group_top[lane + 64 * i];
      int32_t lo = kNoScore + 1, hi = 32768;  // n groups or all reach lo, fewer hi
      while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        int32_t c = 0;
#pragma unroll
        for (int i = 0; i < GROUPS / 64; ++i) c += __popcll(__ballot(g[i] >= mid));
        if (c >= n_top) lo = mid;
        else hi = mid;
      }
      if (lane == 0) bound = lo;
    }
    __syncthreads();
    int32_t least = bound, ties = INT32_MIN, turn = 0;
    for (;;) {
      // every score not below `least`: few units have one
#pragma unroll
      for (int k = 0; k < U; ++k) {
        s16x2 m = pair(s[k][0]);
#pragma unroll
        for (int j = 1; j < 4; ++j) m = __builtin_elementwise_max(m, pair(s[k][j]));
        if (max((int32_t)m.x, (int32_t)m.y) < least) continue;
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          hits |= (uint32_t)((int32_t)(int16_t)(s[k][j >> 1] >> (16 * (j & 1))) >= least) << j;
        while (hits) {
          const int32_t j = __ffs(hits) - 1;
          hits &= hits - 1;
          const uint32_t w = j < 4 ? (j < 2 ? s[k][0] : s[k][1]) : (j < 6 ? s[k][2] : s[k][3]);
          const int32_t at = atomicAdd(&count, 1);
          if (at < CAP)
            list[at] = key_of((int16_t)(w >> (16 * (j & 1))), v0 + (tid + k * NT) * 8 + j - off);
        }
      }
      __syncthreads();
      // (A short row has fewer groups: 64 best of 400 scores, ranked among all 400, took
      // 25 us, searched 12.)
      if (ties != INT32_MIN || count <= (U == 1 ? 2 * MAXN : CAP)) break;
      // More than that: the n-th largest score itself. At least n scores are not below
      // lo, fewer than n are not below hi.
      int32_t lo = kNoScore + 1, hi = 32768;
      while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        int32_t c = 0;
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
          for (int j = 0; j < 8; ++j) c += (int32_t)(int16_t)(s[k][j >> 1] >> (16 * (j & 1))) >= mid;
        c = (int32_t)scalar_sum((uint32_t)c);
        turn ^= 1;  // (the other counts may still be read)
        if (lane == 0) tally[turn][wave] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) c += tally[turn][i];
        if (c >= n_top) lo = mid;
        else hi = mid;
      }
      __syncthreads();
      if (tid == 0) count = 0;
      __syncthreads();
      ties = lo;
      least = hi;  // (32768: none)
    }
    if (ties != INT32_MIN) {
      const int32_t lo = ties;
      // the first of those that equal the n-th largest, in the order of their index
      int32_t have = count;
#pragma unroll 1
      for (int k = 0; k < U && have < n_top; ++k) {
        int32_t mine = 0;
        u32x4 w = s[0];
#pragma unroll
        for (int i = 1; i < U; ++i) w = i == k ? s[i] : w;
#pragma unroll
        for (int j = 0; j < 8; ++j) mine += (int32_t)(int16_t)(w[j >> 1] >> (16 * (j & 1))) == lo;
        int32_t before = mine;  // of the wave's lanes up to this one
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int32_t u = __shfl_up(before, o, 64);
          before += lane >= o ? u : 0;
        }
        __syncthreads();
        if (lane == 63) tally[0][wave] = before;
        __syncthreads();
        int32_t at = have + before - mine;
        for (int i = 0; i < WAVES; ++i) {
          at += i < wave ? tally[0][i] : 0;
          have += tally[0][i];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if ((int32_t)(int16_t)(w[j >> 1] >> (16 * (j & 1))) == lo) {
            if (at < n_top) list[at] = key_of(lo, v0 + (tid + k * NT) * 8 + j - off);
            ++at;
          }
      }
      __syncthreads();
      if (tid == 0) count = min(have, n_top);
      __syncthreads();
    }
  } else {
    __syncthreads();
  }

  uint64_t L = 0, B = 0;
  if (MODE != BEST) {
#pragma unroll
    for (int i = 0; i < WAVES; ++i) L += wave_sum[i][0], B += wave_sum[i][1];
  }
  const int64_t at = row * P + part;
  if (MODE == SUMS) {
    if (tid == 0) ws.sums[2 * at] = L, ws.sums[2 * at + 1] = B;
    return;
  }
  int32_t lg = 0;
  if (MODE == ALL) {
    if (tid == 0) {
      lg = L ? log2_q16(L) : 0;
      lg_shared = lg;
      a.entropy[row] = L ? entropy_q16(lg, L, B) : 0;
    }
    __syncthreads();
    lg = lg_shared;
    write_given(a, row, top, lg, tid, NT);
  } else if (tid == 0) {
    ws.top[at] = top;
  }
  if (n_top == 0) return;
  const int32_t n = count;
  // a key's rank is the number of larger ones: 16 lanes count them
  for (int32_t i0 = 0; i0 < n; i0 += NT / 16) {
    const int32_t i = i0 + tid / 16;
    const unsigned long long key = i < n ? list[i] : 0;
    int32_t rank = 0;
#pragma unroll 4
    for (int32_t j = tid & 15; j < n; j += 16) rank += list[j] > key;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) rank += __shfl_xor(rank, o, 64);
    if (i >= n || rank >= n_top || (tid & 15)) continue;
    if (MODE == ALL) {
      a.top[row * n_top + rank] = key_index(key);
      a.top_lp[row * n_top + rank] = log_prob(key_score(key), top, lg);
    } else {
      ws.keys[at * n_top + rank] = key;
    }
  }
  for (int32_t i = n + tid; i < n_top; i += NT) {
    if (MODE == ALL) {
      a.top[row * n_top + i] = -1;
      a.top_lp[row * n_top + i] = kNoLogProb;
    } else {
      ws.keys[at * n_top + i] = 0;
    }
  }
}

constexpr int JOIN = 512;

// The parts of a row joined.
__global__ __launch_bounds__(JOIN) void log_probs_join_kernel(LogProbArgs a, PartView ws, int32_t P) {
  __shared__ unsigned long long keys[MAXP * MAXN];
  __shared__ int32_t have;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int32_t n = a.n_top;
  const int32_t lane = tid & 63;  // (at most 64 parts)
  const int32_t top = wave_max_i32(lane < P ? ws.top[row * P + lane] : kNoScore);
  const uint64_t L = wave_sum_u64(lane < P ? ws.sums[2 * (row * P + lane)] : 0),
                 B = wave_sum_u64(lane < P ? ws.sums[2 * (row * P + lane) + 1] : 0);
  int32_t mine = 0;
  if (tid == 0) have = 0;
  for (int32_t i = tid; i < P * n; i += JOIN) {
    keys[i] = ws.keys[row * P * n + i];
    mine += keys[i] != 0;
  }
  const int32_t lg = L ? log2_q16(L) : 0;
  if (tid == 0) a.entropy[row] = L ? entropy_q16(lg, L, B) : 0;
  write_given(a, row, top, lg, tid, JOIN);
  __syncthreads();
  if (mine) atomicAdd(&have, mine);
  // a key's rank: the larger keys of each part's sorted list (keys differ, but for 0),
  // four lanes a key
  for (int32_t i0 = 0; i0 < P * n; i0 += JOIN / 4) {
    const int32_t i = i0 + tid / 4;
    const unsigned long long key = i < P * n ? keys[i] : 0;
    int32_t rank = 0;
    if (key)
      for (int32_t p = tid & 3; p < P; p += 4) {
        int32_t lo = 0, hi = n;  // keys[p][lo - 1] > key >= keys[p][hi]
        while (lo < hi) {
          const int32_t mid = (lo + hi) >> 1;
          if (keys[p * n + mid] > key) lo = mid + 1;
          else hi = mid;
        }
        rank += lo;
      }
    rank += __shfl_xor(rank, 1, 64);
    rank += __shfl_xor(rank, 2, 64);
    if (key == 0 || rank >= n || (tid & 3)) continue;
    a.top[row * n + rank] = key_index(key);
    a.top_lp[row * n + rank] = log_prob(key_score(key), top, lg);
  }
  __syncthreads();
  for (int32_t i = have + tid; i < n; i += JOIN) {  // fewer scores than n in all parts
    a.top[row * n + i] = -1;
    a.top_lp[row * n + i] = kNoLogProb;
  }
}

// Parts of a row: one up to the scores that a workgroup keeps.  (16 rows of 100003
// scores, 20 best: 15 us; in 12 parts of two launches 29.)
int32_t parts_of(const LogProbArgs& a) {
  constexpr int32_t most = 1024 * 14 * 8 - 16, part = 1024 * 8 * 8 - 16;
  return a.V <= most ? 1 : (a.V + part - 1) / part;
}

PartView carve(const LogProbArgs& a, int32_t P, void* ws) {
  const int64_t n = a.rows * P;
  int8_t* w = (int8_t*)ws;
  PartView v = {};
  if (!w) return v;
  v.sums = (unsigned long long*)w;
  v.keys = v.sums + 2 * n;
  v.top = (int32_t*)(v.keys + n * a.n_top);
  return v;
}

// The workgroup, by the units of a row and by how many rows there are: threads keep 1
// to 14 units.  Many rows take smaller workgroups, of which a CU has several, so that
// one loads while another sums; few rows take more threads each.  In us, without
// alternatives:
//   2048 rows of 9000: 256 x 8 17.2, 512 x 4 20.3, 1024 x 2 41.7; 200 rows of 12000:
//     256 x 8 6.2, 512 x 4 6.0, 1024 x 2 6.5.
//   512 rows of 30000: 512 x 8 11.9, 1024 x 4 15.5; 200 rows of 32000, 8 best: 512 x 8
//     10.1, 1024 x 4 9.8.
//   400 rows of 50000: 512 x 14 15.9, 1024 x 8 20.9.
template <int MODE>
hipError_t launch_mode(const LogProbArgs& a, const PartView& v, int32_t P, hipStream_t s) {
  const dim3 grid((unsigned)(a.rows * P));
  const int32_t units = (a.V + P - 1) / P / 8 + 2;  // of a part, wherever it starts
  const auto go = [&](auto nt, auto u) {
    constexpr int NT = decltype(nt)::value, U = decltype(u)::value;
    hipLaunchKernelGGL((log_probs_kernel<NT, U, MODE>), grid, dim3(NT), 0, s, a, v, P);
    return hipGetLastError();
  };
  if constexpr (MODE == ALL) {
    if (units <= 256) return go(IntC<256>{}, IntC<1>{});
    if (units <= 256 * 4) return go(IntC<256>{}, IntC<4>{});
    if (units <= 256 * 8 && a.rows > 1024) return go(IntC<256>{}, IntC<8>{});
    if (units <= 512 * 4) return go(IntC<512>{}, IntC<4>{});
    if (units <= 512 * 8 && a.rows > 256) return go(IntC<512>{}, IntC<8>{});
    if (units <= 1024 * 4) return go(IntC<1024>{}, IntC<4>{});
    if (units <= 512 * 14 && a.rows > 256) return go(IntC<512>{}, IntC<14>{});
    if (units > 1024 * 8) return go(IntC<1024>{}, IntC<14>{});
  }
  return go(IntC<1024>{}, IntC<8>{});  // (every part: see parts_of)
}

}  // namespace

bool log_probs_fits(const LogProbArgs& a) {
  return a.rows < (int64_t)1 << 22 && a.rows * parts_of(a) < (int64_t)1 << 22;  // of 1024 threads
}

size_t log_probs_workspace(const LogProbArgs& a) {
  const int32_t P = parts_of(a);
  return P <= 1 ? 0 : (size_t)a.rows * P * (20 + 8 * (size_t)a.n_top);
}

hipError_t launch_log_probs(const LogProbArgs& a, void* ws, hipStream_t s) {
  const int32_t P = parts_of(a);
  const PartView v = carve(a, P, P > 1 ? ws : nullptr);
  if (P == 1) return launch_mode<ALL>(a, v, P, s);
  hipError_t e = launch_mode<BEST>(a, v, P, s);
  if (e == hipSuccess) e = launch_mode<SUMS>(a, v, P, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(log_probs_join_kernel, dim3((unsigned)a.rows), dim3(JOIN), 0, s, a, v, P);
  return hipGetLastError();
}

}  // namespace ilw
