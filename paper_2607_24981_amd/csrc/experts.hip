// experts.hip -- routing of tokens to experts, and the experts' rows back to tokens.
//
// Routing: int16 scores in 1/64 octave become probabilities in 2^-30 (softmax or
// sigmoid, 2^(-a/64) from a table of 64 values), the choice goes by probability +
// bias within the groups that are kept, and the (token, choice) pairs are sorted by
// expert, then by token.
//   choose_kernel  a wave a token: probabilities, groups, the best top_k; a
//                  workgroup of 64 tokens counts its choices of each expert
//   place_kernel   each workgroup sums the counts of the workgroups before it and
//                  all of them, which gives every expert's start, and places its 64
//                  tokens: the rank of a token among those of the workgroup that
//                  chose an expert is a popcount of the expert's 64-bit set
// 64 tokens or fewer are chosen and placed by one workgroup in one launch.  No
// counter is shared between workgroups: the order does not depend on their timing.
#include "step_internal.h"

namespace ilw {
namespace {

constexpr int NT = 256, WAVES = NT / 64;
constexpr int TB = 64;  // tokens a workgroup

// Probabilities of the NV scores a lane has (experts lane + 64 i) in 2^-30.
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
  top = wave_max_i32(top);
  uint64_t sum = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    p[i] = s[i] == kNoScore ? 0 : exp2_q30(table, (uint32_t)(top - s[i]));
    sum += p[i];
  }
  sum = wave_sum_u64(sum);
  if (sum == 0) return;  // no expert to be had
  const int32_t d = bit_length(sum) - 31;
  const uint32_t f = inverse_2p62((uint32_t)(sum >> d));
#pragma unroll
  for (int i = 0; i < NV; ++i) p[i] = __umulhi(p[i], f) >> d;
}

// Leaves in c (INT32_MIN: none) only the experts of the top_groups best groups.
// `best` is the wave's LDS for E values.
template <int NV>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, int32_t (&c)[NV], int32_t* best,
                                            int lane) {
  const int32_t per = a.E / a.groups;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (lane + 64 * i < a.E) best[lane + 64 * i] = c[i];
  __builtin_amdgcn_wave_barrier();
  // a group is a lane's: its best one or two
  int32_t b0 = INT32_MIN, b1 = INT32_MIN;
  if (lane < a.groups)
    for (int32_t i = 0; i < per; ++i) {
      const int32_t v = best[lane * per + i];
      b1 = max(b1, min(b0, v));
      b0 = max(b0, v);
    }
  __builtin_amdgcn_wave_barrier();
  const int64_t score =
      b0 == INT32_MIN ? INT64_MIN : (int64_t)b0 + (a.group_best == 2 && b1 != INT32_MIN ? b1 : 0);
  int32_t rank = 0;
  for (int32_t g = 0; g < a.groups; ++g) {
    const int64_t other = (int64_t)(((uint64_t)(uint32_t)__shfl((int32_t)(score >> 32), g, 64) << 32) |
                                    (uint32_t)__shfl((int32_t)score, g, 64));
    rank += other > score || (other == score && g < lane);
  }
  const uint64_t kept = __ballot(lane < a.groups && b0 != INT32_MIN && rank < a.top_groups);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int32_t e = lane + 64 * i;
    if (e < a.E && !(kept >> (e / per) & 1)) c[i] = INT32_MIN;
  }
}

// The choices of token t: writes expert and weight, enters them in the sets.
template <int NV>
__device__ __forceinline__ void choose(const RouteArgs& a, int32_t t, int32_t bit, int lane,
                                       const uint32_t* table, int32_t* best,
                                       unsigned long long* sets) {
  int32_t s[NV], c[NV];
  uint32_t p[NV];
  const int16_t* row = a.logits + (int64_t)t * a.ld;
#pragma unroll
  for (int i = 0; i < NV; ++i) s[i] = lane + 64 * i < a.E ? row[lane + 64 * i] : kNoScore;
  probabilities<NV>(s, p, a.sigmoid, table);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int32_t e = lane + 64 * i;
    const int32_t b = a.bias && e < a.E ? min(max(a.bias[e], -(1 << 30)), 1 << 30) : 0;
    c[i] = s[i] == kNoScore ? INT32_MIN : (int32_t)p[i] + b;
  }
  if (a.groups > 1) keep_groups<NV>(a, c, best, lane);
  int32_t expert = -1;  // lane j: choice j
  uint32_t prob = 0;
  for (int32_t j = 0; j < a.top_k; ++j) {
    int32_t m = c[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) m = max(m, c[i]);
    m = wave_max_i32(m);
    if (m == INT32_MIN) break;
    bool found = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint64_t hit = __ballot(c[i] == m);
      if (!found && hit) {
        found = true;
        const int l = __ffsll((unsigned long long)hit) - 1;
        const uint32_t pj = __builtin_amdgcn_readlane(p[i], l);
        if (lane == l) c[i] = INT32_MIN;
        if (lane == j) {
          expert = l + 64 * i;
          prob = pj;
        }
      }
    }
  }
  uint32_t r = prob;
  if (a.renorm) {
    const uint64_t sum = wave_sum_u64(prob);
    const int32_t n = bit_length(sum);
    if (sum) {
      const uint32_t unit = (uint32_t)(n <= 31 ? sum << (31 - n) : sum >> (n - 31));
      r = (uint32_t)(((uint64_t)prob * inverse_2p62(unit)) >> (n + 1));
    }
  }
  if (lane < a.top_k) {
    const int64_t w = ((int64_t)((uint64_t)r * (uint32_t)a.mult) + ((int64_t)1 << (a.shift - 1))) >> a.shift;
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
    const int32_t n = e0 + lane < E ? total[e0 + lane] : 0;
    int32_t v = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int32_t u = __shfl_up(v, o, 64);
      v += lane >= o ? u : 0;
    }
    if (e0 + lane < E) total[e0 + lane] = before + v - n;
    before += __shfl(v, 63, 64);
  }
  return before;
}

// Places the workgroup's tokens: start[e] is the row of its first token of expert e.
__device__ __forceinline__ void place(const RouteArgs& a, int32_t t0, const int32_t* start,
                                      const unsigned long long* sets, const int32_t* expert) {
  const int32_t n = min(TB, a.T - t0) * a.top_k;
  for (int32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const int64_t at = (int64_t)t0 * a.top_k + i;
    const int32_t e = expert[at], t = i / a.top_k;
    int32_t slot = -1;
    if (e >= 0) {
      slot = start[e] + __popcll(sets[e] & (((unsigned long long)1 << t) - 1));
      a.rows[slot] = t0 + t;
    }
    a.slot[at] = slot;
  }
}

template <int NV, bool ONE>
__global__ __launch_bounds__(NT) void choose_kernel(RouteArgs a, uint8_t* counts) {
  __shared__ uint32_t table[64];
  __shared__ unsigned long long sets[64 * NV];
  __shared__ int32_t best[WAVES][64 * NV];
  __shared__ int32_t used;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t t0 = blockIdx.x * TB, n = min(TB, a.T - t0);
  load_exp2(table);
  for (int32_t e = tid; e < a.E; e += NT) sets[e] = 0;
  __syncthreads();
  for (int32_t t = wave; t < n; t += WAVES)
    choose<NV>(a, t0 + t, t, lane, table, best[wave], sets);
  __syncthreads();
  if (!ONE) {
    for (int32_t e = tid; e < a.E; e += NT)
      counts[(int64_t)blockIdx.x * a.E + e] = (uint8_t)__popcll(sets[e]);
    return;
  }
  int32_t* start = best[0];
  for (int32_t e = tid; e < a.E; e += NT) start[e] = __popcll(sets[e]);
  __syncthreads();
  if (wave == 0) {
    const int32_t all = starts(start, a.E, lane);
    if (lane == 0) used = a.offsets[a.E] = all;
  }
  __syncthreads();
  for (int32_t e = tid; e < a.E; e += NT) a.offsets[e] = start[e];
  place(a, t0, start, sets, a.expert);  // (this workgroup's own stores, before barriers)
  for (int32_t i = used + tid; i < a.T * a.top_k; i += NT) a.rows[i] = -1;
}

constexpr int MAXE = 1024;

__global__ __launch_bounds__(NT) void place_kernel(RouteArgs a, const uint8_t* counts) {
  __shared__ unsigned long long sets[MAXE];
  __shared__ int32_t start[MAXE];
  __shared__ int32_t used;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t b = blockIdx.x, nb = gridDim.x, t0 = b * TB;
  int32_t before[MAXE / NT];
#pragma unroll
  for (int i = 0; i < MAXE / NT; ++i) {
    const int32_t e = tid + i * NT;
    before[i] = 0;
    if (e < a.E) {
      int32_t all = 0;
      for (int32_t k = 0; k < nb; ++k) {
        const int32_t c = counts[(int64_t)k * a.E + e];
        before[i] += k < b ? c : 0;
        all += c;
      }
      sets[e] = 0;
      start[e] = all;
    }
  }
  __syncthreads();
  if (wave == 0) {
    const int32_t all = starts(start, a.E, lane);
    if (lane == 0) used = all;
  }
  const int32_t n = min(TB, a.T - t0) * a.top_k;
  for (int32_t i = tid; i < n; i += NT) {
    const int32_t e = a.expert[(int64_t)t0 * a.top_k + i];
    if (e >= 0) atomicOr(&sets[e], 1ull << (i / a.top_k));
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MAXE / NT; ++i) {
    const int32_t e = tid + i * NT;
    if (e < a.E) {
      if (b == 0) a.offsets[e] = start[e];
      start[e] += before[i];
    }
  }
  if (b == 0 && tid == 0) a.offsets[a.E] = used;
  __syncthreads();
  place(a, t0, start, sets, a.expert);
  const int64_t all = (int64_t)a.T * a.top_k;
  for (int64_t i = used + (int64_t)b * NT + tid; i < all; i += (int64_t)nb * NT) a.rows[i] = -1;
}

// ------------------------------------------------------------------- combine
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A wave has 64 units of 16 bytes of a token's row.
template <int BYTES>
__global__ __launch_bounds__(NT) void combine_kernel(CombineArgs a, int32_t parts) {
  constexpr int VALS = 16 / BYTES, lim = BYTES == 1 ? 127 : 32767;
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = wave / parts;
  const int32_t unit = (int32_t)(wave - t * parts) * 64 + lane;
  const int64_t ld = (int64_t)a.N * BYTES;
  if (t >= a.T || unit * VALS >= a.N) return;
  int64_t sum[VALS];
#pragma unroll
  for (int i = 0; i < VALS; ++i) sum[i] = 0;
  const auto value = [](const u32x4& w, int i) {
    return BYTES == 1 ? (int32_t)(int8_t)(w[i >> 2] >> (8 * (i & 3)))
                      : (int32_t)(int16_t)(w[i >> 1] >> (16 * (i & 1)));
  };
  for (int32_t j = 0; j < a.top_k; ++j) {
    const int64_t s = a.slot[t * a.top_k + j];
    const int32_t w = a.weight[t * a.top_k + j];
    if ((uint64_t)s >= (uint64_t)a.v_rows) continue;
    const u32x4 v = *(const u32x4*)((const int8_t*)a.v + s * ld + unit * 16);
#pragma unroll
    for (int i = 0; i < VALS; ++i) sum[i] += (int64_t)w * value(v, i);
  }
  u32x4 skip = {0, 0, 0, 0}, out;
  if (a.skip) skip = *(const u32x4*)((const int8_t*)a.skip + t * ld + unit * 16);
  int32_t y[VALS];
#pragma unroll
  for (int i = 0; i < VALS; ++i) {
    const int64_t u = min(max((sum[i] + 128) >> 8, -(int64_t)INT32_MAX), (int64_t)INT32_MAX);
    const int64_t v = (u * a.mult_a + (int64_t)value(skip, i) * a.mult_b +
                       ((int64_t)1 << (a.shift - 1))) >> a.shift;
    y[i] = (int32_t)min(max(v, (int64_t)-lim), (int64_t)lim);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    out[k] = BYTES == 1 ? pack4(y[4 * k % VALS], y[(4 * k + 1) % VALS], y[(4 * k + 2) % VALS],
                                y[(4 * k + 3) % VALS])
                        : __builtin_amdgcn_perm((uint32_t)y[(2 * k + 1) % VALS],
                                                (uint32_t)y[2 * k % VALS], 0x05040100u);
  *(u32x4*)((int8_t*)a.y + t * ld + unit * 16) = out;
}

int32_t combine_parts(const CombineArgs& a) { return (a.N * (a.bits / 8) / 16 + 63) / 64; }

}  // namespace

size_t route_workspace(int32_t T, int32_t E) {
  const int64_t blocks = ((int64_t)T + TB - 1) / TB;
  return blocks <= 1 ? 0 : (size_t)(blocks * E);
}

hipError_t launch_route(const RouteArgs& a, void* ws, hipStream_t s) {
  const int32_t blocks = a.T > 0 ? (a.T - 1) / TB + 1 : 1;  // (no token: offsets of 0)
  uint8_t* counts = (uint8_t*)ws;
  const auto choose_with = [&](auto nv) {
    constexpr int NV = decltype(nv)::value;
    if (blocks == 1)
      hipLaunchKernelGGL((choose_kernel<NV, true>), dim3(1), dim3(NT), 0, s, a, counts);
    else
      hipLaunchKernelGGL((choose_kernel<NV, false>), dim3(blocks), dim3(NT), 0, s, a, counts);
  };
  if (a.E <= 64) choose_with(IntC<1>{});
  else if (a.E <= 128) choose_with(IntC<2>{});
  else if (a.E <= 256) choose_with(IntC<4>{});
  else if (a.E <= 512) choose_with(IntC<8>{});
  else choose_with(IntC<16>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || blocks == 1) return e;
  hipLaunchKernelGGL(place_kernel, dim3(blocks), dim3(NT), 0, s, a, counts);
  return hipGetLastError();
}

bool combine_fits(const CombineArgs& a) {
  return (a.T * combine_parts(a) + WAVES - 1) / WAVES < (int64_t)1 << 24;
}

hipError_t launch_combine(const CombineArgs& a, hipStream_t s) {
  const int32_t parts = combine_parts(a);
  const int64_t blocks = (a.T * parts + WAVES - 1) / WAVES;
  if (a.bits == 8)
    hipLaunchKernelGGL((combine_kernel<1>), dim3((unsigned)blocks), dim3(NT), 0, s, a, parts);
  else
    hipLaunchKernelGGL((combine_kernel<2>), dim3((unsigned)blocks), dim3(NT), 0, s, a, parts);
  return hipGetLastError();
}

}  // namespace ilw
