// experts.hip -- routing of tokens to experts, and the experts' rows back to tokens.
//
// Routing: int16 scores in 1/64 octave become probabilities in 2^-30 (softmax or
// sigmoid, 2^(-a/64) from a table of 64 values), the choice goes by probability +
// bias within the groups that are kept, and the (token, choice) pairs are sorted by
// expert, then by token.
//   choose_kernel  a wave a token, NV neighbouring experts a lane, sorted there; the
//                  best is found top_k times: the largest of the lanes' first by DPP,
//                  then the lowest lane that has it, which is the lowest index
//   place_kernel   each workgroup sums the counts of the workgroups before it and
//                  all of them, which gives every expert's start, and places its
//                  tokens 64 at a time: the rank of a token among the 64 that chose
//                  an expert is a popcount of the expert's 64-bit set
// A few tokens are chosen and placed by one workgroup in one launch.  At most MAXB
// workgroups share the tokens, so that the counts they all read stay few.  No
// counter is shared between workgroups: the order does not depend on their timing.
//
// Bound: vector instructions of choose_kernel, about 570 a token of 256 experts and 8
// choices in groups (16384 tokens: 20 us of 26.6; a lane's experts sorted once, maxima
// by DPP; found over all experts again for each choice, through LDS, both launches took
// 150), then place_kernel, whose workgroups read all counts (6 us).  A few tokens are
// bound by the launch (32 tokens of 64 experts: 5.4 us on the device).
#include "step_internal.h"

namespace ilw {
namespace {

constexpr int SET = 64;    // tokens that place_kernel places at a time
constexpr int MAXB = 256;  // workgroups of choose_kernel
constexpr int MAXE = 1024;
constexpr int NT = 1024;   // threads of place_kernel

// How choose_kernel shares the tokens: `waves` a workgroup, which takes `sets` sets of
// `tokens` tokens one after another and counts them together.
struct Share {
  int32_t waves, tokens, sets, blocks;
};

// Probabilities of a lane's NV scores in 2^-30.
template <int NV>
__device__ __forceinline__ void probabilities(const int32_t (&s)[NV], uint32_t (&p)[NV],
                                              bool sigmoid, const uint32_t* table) {
  if (sigmoid) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t t = exp2_q30(table, (uint32_t)abs(s[i]));
      const uint32_t f = inverse_2p62((1u << 30) + t);
      p[i] = s[i] == kNoScore ? 0 : __umulhi(s[i] < 0 ? t : 1u << 30, f);
    }
    return;
  }
  int32_t top = kNoScore;
#pragma unroll
  for (int i = 0; i < NV; ++i) top = max(top, s[i]);
  top = scalar_max(top);
  uint64_t sum = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    p[i] = s[i] == kNoScore ? 0 : exp2_q30(table, (uint32_t)(top - s[i]));
    sum += p[i];
  }
  sum = scalar_sum_u64(sum);
  if (sum == 0) return;  // no expert to be had
  const int32_t d = bit_length(sum) - 31;
  const uint32_t f = inverse_2p62((uint32_t)(sum >> d));
#pragma unroll
  for (int i = 0; i < NV; ++i) p[i] = __umulhi(p[i], f) >> d;
}

// A score and its lane's index of it, ordered by score, then by lower index.
struct Scored {
  int32_t c, i;
};
__device__ __forceinline__ int64_t order_of(const Scored& x) {
  return (int64_t)(((uint64_t)(uint32_t)x.c << 32) | (uint32_t)~x.i);
}
// Best first, by odd-even merging.
template <int NV>
__device__ __forceinline__ void sort_lane(Scored (&x)[NV]) {
#pragma unroll
  for (int p = 1; p < NV; p <<= 1)
#pragma unroll
    for (int k = p; k >= 1; k >>= 1)
#pragma unroll
      for (int j = k % p; j + k < NV; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i) {
          const int l = j + i, r = j + i + k;
          if (r < NV && l / (2 * p) == r / (2 * p)) {
            const bool swap = order_of(x[l]) < order_of(x[r]);
            const Scored u = swap ? x[r] : x[l], v = swap ? x[l] : x[r];
            x[l] = u;
            x[r] = v;
          }
        }
}

template <int NV>
struct Order {
  typedef uint32_t type;
};
template <>
struct Order<16> {
  typedef uint64_t type;
};

// How the groups lie on the lanes.  Where a group is a power of two of whole lanes
// (`span` of them), its best two come out of the lanes' own; else `sub` lanes, a power
// of two, go over a group's experts in LDS.
template <int NV>
struct Groups {
  int32_t per, span, sub, log_sub;
  float inv_per;
  __device__ __forceinline__ void init(const RouteArgs& a) {
    per = a.E / a.groups;
    span = per % NV == 0 && ((per / NV) & (per / NV - 1)) == 0 ? per / NV : 0;
    log_sub = span ? 31 - __clz(span) : 6 - (32 - __clz(a.groups - 1));  // groups > 1
    sub = 1 << log_sub;
    inv_per = 1.f / (float)per;
  }
};

// Leaves in x (INT32_MIN: none) only the experts of the top_groups best groups.
// `lds` is the wave's, for E values; x is sorted and stays so where span > 0.
template <int NV>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, const Groups<NV>& g,
                                            Scored (&x)[NV], int32_t* lds, int lane) {
  const int32_t group = lane >> g.log_sub;
  int32_t b0 = INT32_MIN, b1 = INT32_MIN;  // the best two
  if (g.span) {
    b0 = x[0].c;
    if (NV > 1) b1 = x[NV > 1 ? 1 : 0].c;
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) lds[lane * NV + x[i].i] = x[i].c;
    __builtin_amdgcn_wave_barrier();
    if (group < a.groups)
      for (int32_t i = lane & (g.sub - 1); i < g.per; i += g.sub) {
        const int32_t v = lds[group * g.per + i];
        b1 = max(b1, min(b0, v));
        b0 = max(b0, v);
      }
    __builtin_amdgcn_wave_barrier();
  }
  const auto merge = [&](int32_t o0, int32_t o1) {
    b1 = max(max(b1, o1), min(b0, o0));
    b0 = max(b0, o0);
  };
  // lanes 1, 2, 4, 8 apart (mirrors do for 4 and 8: quads and halves are alike by then)
  if (g.sub > 1) merge(dpp_or<0xb1, 0xf>(0, b0), dpp_or<0xb1, 0xf>(0, b1));
  if (g.sub > 2) merge(dpp_or<0x4e, 0xf>(0, b0), dpp_or<0x4e, 0xf>(0, b1));
  if (g.sub > 4) merge(dpp_or<0x141, 0xf>(0, b0), dpp_or<0x141, 0xf>(0, b1));
  if (g.sub > 8) merge(dpp_or<0x140, 0xf>(0, b0), dpp_or<0x140, 0xf>(0, b1));
  for (int32_t o = 16; o < g.sub; o <<= 1) merge(__shfl_xor(b0, o, 64), __shfl_xor(b1, o, 64));
  const int64_t score =
      b0 == INT32_MIN ? INT64_MIN : (int64_t)b0 + (a.group_best == 2 && b1 != INT32_MIN ? b1 : 0);
  int32_t rank = 0;
  for (int32_t h = 0; h < a.groups; ++h) {
    const int32_t l = h << g.log_sub;
    const int64_t other =
        (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int32_t)(score >> 32), l) << 32) |
                  (uint32_t)__builtin_amdgcn_readlane((int32_t)score, l));
    rank += other > score || (other == score && h < group);
  }
  const bool stays = group < a.groups && b0 != INT32_MIN && rank < a.top_groups;
  if (g.span) {
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i].c = stays ? x[i].c : INT32_MIN;
    return;
  }
  const uint64_t kept = __ballot(stays);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int32_t h = min(fdiv(lane * NV + x[i].i, g.per, g.inv_per), a.groups - 1);
    x[i].c = (kept >> (h << g.log_sub)) & 1 ? x[i].c : INT32_MIN;
  }
  sort_lane<NV>(x);
}

// The choices of token t: writes expert and weight, enters them in the sets.
template <int NV>
__device__ __forceinline__ void choose(const RouteArgs& a, const Groups<NV>& g,
                                       const int32_t* bias, int32_t t, int32_t bit, int lane,
                                       const uint32_t* table, int32_t* lds,
                                       unsigned long long* sets) {
  int32_t s[NV];
  uint32_t p[NV];
  Scored x[NV];
  const int16_t* row = a.logits + (int64_t)t * a.ld;
#pragma unroll
  for (int i = 0; i < NV; ++i) s[i] = lane * NV + i < a.E ? row[lane * NV + i] : kNoScore;
  probabilities<NV>(s, p, a.sigmoid, table);
#pragma unroll
  for (int i = 0; i < NV; ++i) x[i] = {s[i] == kNoScore ? INT32_MIN : (int32_t)p[i] + bias[lane * NV + i], i};
  sort_lane<NV>(x);
  if (a.groups > 1) keep_groups<NV>(a, g, x, lds, lane);
#pragma unroll
  for (int i = 0; i < NV; ++i) lds[lane * NV + i] = (int32_t)p[i];
  __builtin_amdgcn_wave_barrier();
  // the lane's order, four bits an expert, so that the next one is a shift away
  typedef typename Order<NV>::type order_t;
  order_t order = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) order |= (order_t)x[i].i << (4 * i);
  int32_t expert = -1;  // lane j: choice j
  for (int32_t j = 0; j < a.top_k; ++j) {
    const int32_t best = scalar_max(x[0].c);
    if (best == INT32_MIN) break;
    const int l = __ffsll((unsigned long long)__ballot(x[0].c == best)) - 1;
    const int32_t e = l * NV + (__builtin_amdgcn_readlane((int32_t)order, l) & (NV - 1));
    expert = lane == j ? e : expert;
    const bool mine = lane == l;
    order >>= mine ? 4 : 0;
#pragma unroll
    for (int i = 0; i + 1 < NV; ++i) x[i].c = mine ? x[i + 1].c : x[i].c;
    x[NV - 1].c = mine ? INT32_MIN : x[NV - 1].c;
  }
  const uint32_t prob = expert >= 0 ? (uint32_t)lds[expert] : 0;
  __builtin_amdgcn_wave_barrier();
  uint32_t r = prob;
  if (a.renorm) {
    const uint64_t sum = scalar_sum_u64(prob);
    const int32_t n = bit_length(sum);
    if (sum) {
      const uint32_t unit = (uint32_t)(n <= 31 ? sum << (31 - n) : sum >> (n - 31));
      r = (uint32_t)(((uint64_t)prob * inverse_2p62(unit)) >> (n + 1));
    }
  }
  if (lane < a.top_k) {
    const int64_t w =
        ((int64_t)((uint64_t)r * (uint32_t)a.mult) + ((int64_t)1 << (a.shift - 1))) >> a.shift;
    const int64_t at = (int64_t)t * a.top_k + lane;
    a.expert[at] = expert;
    a.weight[at] = (int32_t)min(w, (int64_t)INT32_MAX);
    if (expert >= 0) atomicOr(&sets[expert], 1ull << bit);
  }
}

// Starts of the experts from their totals, in LDS: total -> start, one wave.
__device__ __forceinline__ int32_t starts(int32_t* total, int32_t E, int lane) {
  int32_t before = 0;
  for (int32_t e0 = 0; e0 < E; e0 += 64) {
    const int32_t n = e0 + lane < E ? total[e0 + lane] : 0, v = wave_scan(n);
    if (e0 + lane < E) total[e0 + lane] = before + v - n;
    before += __builtin_amdgcn_readlane(v, 63);
  }
  return before;
}

// Places 64 tokens from t0 on: start[e] is the row of the first that chose e.
__device__ __forceinline__ void place(const RouteArgs& a, int32_t t0, const int32_t* start,
                                      const unsigned long long* sets) {
  const int32_t n = min(SET, a.T - t0) * a.top_k;
  const float inv_k = 1.f / (float)a.top_k;
  for (int32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const int64_t at = (int64_t)t0 * a.top_k + i;
    const int32_t e = a.expert[at], t = fdiv(i, a.top_k, inv_k);
    int32_t slot = -1;
    if (e >= 0) {
      slot = start[e] + __popcll(sets[e] & (((unsigned long long)1 << t) - 1));
      a.rows[slot] = t0 + t;
    }
    a.slot[at] = slot;
  }
}

// Counts of a workgroup, in whole words.
template <typename C>
__host__ __device__ __forceinline__ int32_t count_stride(int32_t E) {
  constexpr int W = 4 / sizeof(C);
  return (E + W - 1) / W * W;
}

// Workgroup b has the sets b * sets .. b * sets + sets - 1.
template <int NV, int WAVES, bool ONE, typename C>
__global__ __launch_bounds__(64 * WAVES) void choose_kernel(RouteArgs a, C* counts, Share sh) {
  constexpr int CNT = 64 * WAVES;
  __shared__ uint32_t table[64];
  __shared__ unsigned long long sets[64 * NV];
  __shared__ int32_t lds[WAVES][64 * NV], bias[64 * NV], count[ONE ? 1 : 64 * NV];
  __shared__ int32_t used;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  load_exp2(table);
  for (int32_t e = tid; e < 64 * NV; e += CNT) {
    bias[e] = a.bias && e < a.E ? min(max(a.bias[e], -(1 << 30)), 1 << 30) : 0;
    sets[e] = 0;
    if (!ONE) count[e] = 0;
  }
  Groups<NV> g;
  if (a.groups > 1) g.init(a);
  __syncthreads();
  for (int32_t k = 0; k < sh.sets; ++k) {
    const int64_t first = ((int64_t)blockIdx.x * sh.sets + k) * sh.tokens;
    if (first >= a.T && !ONE) break;
    const int32_t t0 = (int32_t)first;
    const int32_t n = min(sh.tokens, a.T - t0);
    for (int32_t t = wave; t < n; t += WAVES)
      choose<NV>(a, g, bias, t0 + t, t, lane, table, lds[wave], sets);
    if (ONE) break;
    __syncthreads();
    for (int32_t e = tid; e < 64 * NV; e += CNT) {
      count[e] += __popcll(sets[e]);
      sets[e] = 0;
    }
    __syncthreads();
  }
  if (!ONE) {
    const int32_t ld = count_stride<C>(a.E);
    for (int32_t e = tid; e < ld; e += CNT)  // (0 behind the experts)
      counts[blockIdx.x * ld + e] = (C)count[e];
    return;
  }
  __syncthreads();
  int32_t* start = lds[0];
  for (int32_t e = tid; e < a.E; e += CNT) start[e] = __popcll(sets[e]);
  __syncthreads();
  if (wave == 0) {
    const int32_t all = starts(start, a.E, lane);
    if (lane == 0) used = a.offsets[a.E] = all;
  }
  __syncthreads();
  for (int32_t e = tid; e < a.E; e += CNT) a.offsets[e] = start[e];
  place(a, 0, start, sets);  // (the workgroup's own stores, before barriers)
  for (int32_t i = used + tid; i < a.T * a.top_k; i += CNT) a.rows[i] = -1;
}

// Workgroup b has the sets of 64 tokens b * per .. b * per + per - 1, whose counts are
// `rows` of the nb rows.
template <typename C>
__global__ __launch_bounds__(NT) void place_kernel(RouteArgs a, const C* counts, int32_t per,
                                                    int32_t rows, int32_t nb) {
  __shared__ unsigned long long sets[MAXE];
  __shared__ int32_t start[MAXE], before[MAXE];
  __shared__ int32_t used;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t b = blockIdx.x;
  const float inv_k = 1.f / (float)a.top_k;
  static_assert(SET * 32 <= 2 * NT, "two choices a thread");
  int32_t x[2];  // a set's choices: loaded, then entered in the sets
  const auto load = [&](int32_t k) {
    const int64_t first = ((int64_t)b * per + k) * SET;
    const int32_t n = first < a.T ? min(SET, a.T - (int32_t)first) * a.top_k : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = tid + i * NT < n ? a.expert[first * a.top_k + tid + i * NT] : -1;
  };
  const auto enter = [&]() {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (x[i] >= 0) atomicOr(&sets[x[i]], 1ull << fdiv(tid + i * NT, a.top_k, inv_k));
  };
  start[tid] = before[tid] = 0;
  sets[tid] = 0;
  __syncthreads();
  // cols threads side by side take a word of W counts each, NT / cols rows at a time
  constexpr int W = 4 / sizeof(C);
  const int32_t words = count_stride<C>(a.E) / W;
  const int32_t lc = words > 1 ? 32 - __clz(words - 1) : 0, cols = 1 << lc;
  const int32_t col = tid & (cols - 1), step = NT >> lc;
  if (col < words) {
    int32_t all[W], mine[W];
#pragma unroll
    for (int i = 0; i < W; ++i) all[i] = mine[i] = 0;
    const uint32_t* c = (const uint32_t*)counts;
#pragma unroll 8
    for (int32_t k = tid >> lc; k < nb; k += step) {
      const uint32_t w = c[k * words + col];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const int32_t v = W == 1 ? (int32_t)w : (int32_t)((w >> (32 / W * i)) & ((1u << (32 / W % 32)) - 1));
        all[i] += v;
        mine[i] += k < b * rows ? v : 0;
      }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (all[i]) atomicAdd(&start[col * W + i], all[i]);  // (whole numbers: in any order)
      if (mine[i]) atomicAdd(&before[col * W + i], mine[i]);
    }
  }
  load(0);
  enter();
  __syncthreads();
  if (wave == 0) {
    const int32_t all = starts(start, a.E, lane);
    if (lane == 0) used = all;
  }
  __syncthreads();
  if (b == 0) {
    if (tid < a.E) a.offsets[tid] = start[tid];
    if (tid == 0) a.offsets[a.E] = used;
  }
  start[tid] += before[tid];
  for (int32_t k = 0; k < per; ++k) {
    const int64_t first = ((int64_t)b * per + k) * SET;
    if (first >= a.T) break;
    const int32_t t0 = (int32_t)first;
    if (k > 0) {
      load(k);
      enter();
    }
    __syncthreads();
    place(a, t0, start, sets);
    if (k + 1 == per) break;
    __syncthreads();
    start[tid] += __popcll(sets[tid]);
    sets[tid] = 0;
    __syncthreads();
  }
  const int64_t all = (int64_t)a.T * a.top_k;
  for (int64_t i = used + (int64_t)b * NT + tid; i < all; i += (int64_t)gridDim.x * NT) a.rows[i] = -1;
}

// ------------------------------------------------------------------- combine
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int CT = 256, CWAVES = CT / 64;

// A thread has a unit of 16 bytes of a token's row.  WHOLE: rows are whole waves of
// units, so that a wave's token, its slots and weights are scalars (8192 tokens of 8 rows
// of 2048 int8 values 33.5 us, numbered through 39.3); else the units of all tokens are
// numbered through and no lane idles (16384 tokens of 8 rows of 64 bytes 6.7 us, 29 with
// a wave a token).  Four choices' rows are on their way at a time.
//
// Bound: bytes (8192 tokens of 8 rows of 2048 int16 values: 65 us, what 336 MB take to
// copy).  int8 rows are summed in 32 bits where the wave's weights are below 2^18 (32
// rows of them stay below 2^31): a 64-bit multiply-add a value takes longer than its
// byte (16384 tokens of 4 rows of 1024 values 24.4 us so, 22.5 in 32 bits).
template <int BYTES, bool WHOLE>
__global__ __launch_bounds__(CT) void combine_kernel(CombineArgs a, int32_t units) {
  constexpr int VALS = 16 / BYTES, lim = BYTES == 1 ? 127 : 32767, AT = 4;
  int64_t t;
  int32_t unit;
  if (WHOLE) {
    const int32_t parts = units / 64;
    const int64_t wave = (int64_t)blockIdx.x * CWAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    t = wave / parts;
    unit = (int32_t)(wave - t * parts) * 64 + (threadIdx.x & 63);
  } else {
    const uint32_t g = blockIdx.x * (uint32_t)CT + threadIdx.x, q = g / (uint32_t)units;
    t = q;
    unit = (int32_t)(g - q * (uint32_t)units);
  }
  if (t >= a.T) return;
  const int64_t ld = (int64_t)a.N * BYTES;
  const int8_t* v = (const int8_t*)a.v + unit * 16;
  const auto value = [](const u32x4& w, int i) {
    return BYTES == 1 ? (int32_t)(int8_t)(w[i >> 2] >> (8 * (i & 3)))
                      : (int32_t)(int16_t)(w[i >> 1] >> (16 * (i & 1)));
  };
  u32x4 skip = {0, 0, 0, 0};
  if (a.skip) skip = *(const u32x4*)((const int8_t*)a.skip + t * ld + unit * 16);
  const int32_t* slot = a.slot + t * a.top_k;
  const int32_t* weight = a.weight + t * a.top_k;
  int32_t y[VALS];
  const auto combine = [&](auto zero) {
    decltype(zero) sum[VALS];
#pragma unroll
    for (int i = 0; i < VALS; ++i) sum[i] = 0;
    if (a.v_rows > 0)
      for (int32_t j0 = 0; j0 < a.top_k; j0 += AT) {
        int64_t s[AT];
        int32_t w[AT];
        u32x4 x[AT];
#pragma unroll
        for (int i = 0; i < AT; ++i) {
          const int32_t j = min(j0 + i, a.top_k - 1);
          s[i] = slot[j];
          w[i] = weight[j];
          // (no such row: the first one, with no weight)
          if ((uint64_t)s[i] >= (uint64_t)a.v_rows) s[i] = w[i] = 0;
        }
#pragma unroll
        for (int i = 0; i < AT; ++i)
          if (j0 + i < a.top_k) x[i] = *(const u32x4*)(v + s[i] * ld);
#pragma unroll
        for (int i = 0; i < AT; ++i) {
          if (j0 + i >= a.top_k) break;
#pragma unroll
          for (int k = 0; k < VALS; ++k) {
            if (sizeof(zero) == 4) sum[k] += __mul24(w[i], value(x[i], k));
            else sum[k] += (int64_t)w[i] * value(x[i], k);
          }
        }
      }
#pragma unroll
    for (int i = 0; i < VALS; ++i) {
      const int64_t u = sizeof(zero) == 4
                            ? ((int64_t)sum[i] + 128) >> 8
                            : min(max(((int64_t)sum[i] + 128) >> 8, -(int64_t)INT32_MAX), (int64_t)INT32_MAX);
      const int64_t r = (u * a.mult_a + (int64_t)value(skip, i) * a.mult_b +
                         ((int64_t)1 << (a.shift - 1))) >> a.shift;
      y[i] = (int32_t)min(max(r, (int64_t)-lim), (int64_t)lim);
    }
  };
  if (BYTES == 1) {
    uint32_t big = 0;
    for (int32_t j = 0; j < a.top_k; ++j) big |= (uint32_t)(weight[j] ^ (weight[j] >> 31));
    if (__all(big < 1u << 18)) combine((int32_t)0);
    else combine((int64_t)0);
  } else {
    combine((int64_t)0);
  }
  u32x4 out;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    out[k] = BYTES == 1 ? pack4(y[4 * k % VALS], y[(4 * k + 1) % VALS], y[(4 * k + 2) % VALS],
                                y[(4 * k + 3) % VALS])
                        : __builtin_amdgcn_perm((uint32_t)y[(2 * k + 1) % VALS],
                                                (uint32_t)y[2 * k % VALS], 0x05040100u);
  *(u32x4*)((int8_t*)a.y + t * ld + unit * 16) = out;
}

// 16-byte units of a row.
int32_t combine_units(const CombineArgs& a) { return a.N * (a.bits / 8) / 16; }

}  // namespace

// A wave a token as long as there are waves: a token takes 2 to 5 us one step after
// the other, and a CU's waves share its issue slots.
// One launch: 32 tokens of 64 experts 5.7 us, in two launches 6.4 (48: 7.2 and 6.7); of
// 256 experts 24 tokens 9.8 and 9.2.  In sets of 64 as from 8192 tokens on, 526 tokens
// of 256 experts took 23.9 us instead of 10.5; 16384 in 512 workgroups of 32, whose
// counts take longer to read, 30.2 instead of 26.6.
static Share share_of(int32_t T, int32_t E) {
  if (T <= 32 && T * E <= 4096) return {16, SET, 1, 1};
  if (T <= 4 * MAXB) return {4, 4, 1, (T + 3) / 4};
  if (T <= 16 * MAXB) return {16, 16, 1, (T + 15) / 16};
  if (T <= 32 * MAXB) return {16, 32, 1, (T + 31) / 32};
  const int32_t sets = ((T - 1) / SET) / MAXB + 1, tokens = SET * sets;
  return {16, SET, sets, (T - 1) / tokens + 1};
}

size_t route_workspace(int32_t T, int32_t E) {
  const int32_t blocks = share_of(T, E).blocks;
  return blocks == 1 ? 0 : (size_t)blocks * E * sizeof(int32_t);
}

template <typename C>
static hipError_t route_with(const RouteArgs& a, C* counts, const Share& sh, hipStream_t s) {
  const dim3 grid(sh.blocks);
  const auto choose_with = [&](auto nv) {
    constexpr int NV = decltype(nv)::value;
    if constexpr (sizeof(C) == 1) {
      if (sh.blocks == 1)
        hipLaunchKernelGGL((choose_kernel<NV, 16, true, C>), grid, dim3(1024), 0, s, a, counts, sh);
      else if (sh.waves == 4)
        hipLaunchKernelGGL((choose_kernel<NV, 4, false, C>), grid, dim3(256), 0, s, a, counts, sh);
    }
    if (sh.blocks > 1 && sh.waves == 16)
      hipLaunchKernelGGL((choose_kernel<NV, 16, false, C>), grid, dim3(1024), 0, s, a, counts, sh);
  };
  if (a.E <= 64) choose_with(IntC<1>{});
  else if (a.E <= 128) choose_with(IntC<2>{});
  else if (a.E <= 256) choose_with(IntC<4>{});
  else if (a.E <= 512) choose_with(IntC<8>{});
  else choose_with(IntC<16>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sh.blocks == 1) return e;
  const int32_t rows = SET > sh.tokens ? SET / sh.tokens : 1;
  hipLaunchKernelGGL((place_kernel<C>), dim3((sh.blocks - 1) / rows + 1), dim3(NT), 0, s, a, counts,
                     sh.sets, rows, sh.blocks);
  return hipGetLastError();
}

// A workgroup's count of an expert is at most its tokens: in a byte up to 255 of them
// (16384 tokens of 256 experts: the counts that every workgroup reads are 64 KB, 6.9 us
// a launch of place_kernel; in 32 bits 8.6).
hipError_t launch_route(const RouteArgs& a, void* ws, hipStream_t s) {
  const Share sh = share_of(a.T, a.E);
  return sh.sets * sh.tokens < 256 ? route_with(a, (uint8_t*)ws, sh, s)
                                   : route_with(a, (int32_t*)ws, sh, s);
}

bool combine_fits(const CombineArgs& a) {
  return a.T < (((int64_t)1 << 32) - CT) / combine_units(a);
}

hipError_t launch_combine(const CombineArgs& a, hipStream_t s) {
  const int32_t units = combine_units(a);
  const dim3 grid((unsigned)((a.T * units + CT - 1) / CT)), block(CT);
  if (a.bits == 8) {
    if (units % 64 == 0) hipLaunchKernelGGL((combine_kernel<1, true>), grid, block, 0, s, a, units);
    else hipLaunchKernelGGL((combine_kernel<1, false>), grid, block, 0, s, a, units);
  } else {
    if (units % 64 == 0) hipLaunchKernelGGL((combine_kernel<2, true>), grid, block, 0, s, a, units);
    else hipLaunchKernelGGL((combine_kernel<2, false>), grid, block, 0, s, a, units);
  }
  return hipGetLastError();
}

}  // namespace ilw
