// step_internal.h -- arguments, launchers and shared arithmetic of the operators
// behind a decoder step's attention: rows quantized with a scale each, linears
// with token and channel scales, routing to experts, their rows combined, log
// probabilities.
#pragma once
#include "ilw_internal.h"

namespace ilw {

constexpr int32_t kNoScore = -32768;        // a score that is not to be had
constexpr int32_t kNoLogProb = INT32_MIN;   // its log probability

struct QuantizeArgs {
  const int16_t* x;
  int64_t ld;  // values between rows
  int8_t* y;
  int32_t* scale;
  int64_t M;
  int32_t K;
};
bool quantize_rows_fits(const QuantizeArgs& a);  // one launch can hold it
hipError_t launch_quantize_rows(const QuantizeArgs& a, hipStream_t s);

struct ScaledArgs {
  const int8_t* x;
  const int32_t* x_scale;
  const int32_t* rows;     // or null
  const int32_t* offsets;  // [E + 1], or null: one expert with every row
  const int8_t* w;
  const int32_t* bias;     // or null
  const int32_t* mult;
  const int32_t* shift;
  void* y;
  int64_t M, x_rows;
  int32_t nq, E, N, K, bits;
};
hipError_t launch_linear_scaled(const ScaledArgs& a, hipStream_t s);

struct RouteArgs {
  const int16_t* logits;
  int64_t ld;
  const int32_t* bias;  // or null
  int32_t* expert;
  int32_t* weight;
  int32_t* offsets;
  int32_t* rows;
  int32_t* slot;
  int32_t T, E, top_k, groups, top_groups, group_best, sigmoid, renorm, mult, shift;
};
size_t route_workspace(int32_t T, int32_t E);
hipError_t launch_route(const RouteArgs& a, void* ws, hipStream_t s);

struct CombineArgs {
  const void* v;
  const int32_t* slot;
  const int32_t* weight;
  const void* skip;  // or null
  void* y;
  int64_t v_rows, T;
  int32_t bits, top_k, N, mult_a, mult_b, shift;
};
bool combine_fits(const CombineArgs& a);  // one launch can hold it
hipError_t launch_combine(const CombineArgs& a, hipStream_t s);

struct LogProbArgs {
  const int16_t* logits;
  int64_t ld;
  const int32_t* given;
  int32_t* given_lp;
  int32_t* entropy;
  int32_t* top;
  int32_t* top_lp;
  int64_t rows;
  int32_t V, n_given, n_top;
};
bool log_probs_fits(const LogProbArgs& a);  // its launches can hold it
size_t log_probs_workspace(const LogProbArgs& a);
hipError_t launch_log_probs(const LogProbArgs& a, void* ws, hipStream_t s);

// 2^(30 - f/64) to the nearest whole number, f in [0, 63].
__device__ constexpr uint32_t kExp2[64] = {
    1073741824u, 1062175491u, 1050733751u, 1039415261u, 1028218693u, 1017142735u, 1006186087u, 995347464u,
    984625594u, 974019220u, 963527098u, 953147997u, 942880699u, 932724001u, 922676710u, 912737649u,
    902905651u, 893179563u, 883558244u, 874040567u, 864625413u, 855311680u, 846098274u, 836984114u,
    827968132u, 819049271u, 810226483u, 801498734u, 792865000u, 784324269u, 775875538u, 767517817u,
    759250125u, 751071493u, 742980960u, 734977579u, 727060411u, 719228525u, 711481005u, 703816941u,
    696235434u, 688735596u, 681316545u, 673977412u, 666717336u, 659535466u, 652430958u, 645402981u,
    638450708u, 631573326u, 624770026u, 618040012u, 611382493u, 604796689u, 598281827u, 591837143u,
    585461881u, 579155293u, 572916640u, 566745190u, 560640218u, 554601009u, 548626854u, 542717053u,
};
// A workgroup's copy of that table, one value a bank.
__device__ __forceinline__ void load_exp2(uint32_t* table) {
  if (threadIdx.x < 64) table[threadIdx.x] = kExp2[threadIdx.x];
}
// 2^(30 - a/64), a >= 0, rounded down past the table's rounding; 0 from 31 octaves on.
__device__ __forceinline__ uint32_t exp2_q30(const uint32_t* table, uint32_t a) {
  a = min(a, 31u * 64u);
  return table[a & 63] >> (a >> 6);
}

// floor((2^62 - 1) / D), exact for D in [2^30, 2^31]: one Newton step on the
// hardware's FP64 reciprocal leaves an error below 2^-13 of a quotient of at most
// 2^32; taken off by 2^-10 its truncation is the quotient or one less (and below 2^32
// for D = 2^30), and the remainder, in [0, 2 D), tells from its 32 bits.
__device__ __forceinline__ uint32_t inverse_2p62(uint32_t D) {
  const double d = (double)D;
  double r = __builtin_amdgcn_rcp(d);
  r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
  const uint32_t q = (uint32_t)__builtin_fma(0x1p62, r, -0x1p-10);
  return q + (~(q * D) >= D);
}

// Wave-wide results in every lane (scalar), by DPP within rows of 16 lanes and from
// row to row: 6 vector instructions where exchanges through LDS take 6 round trips.
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t dpp_or(int32_t old, int32_t v) {
  return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int32_t scalar_max(int32_t v) {
  v = max(v, dpp_or<0x111, 0xf>(INT32_MIN, v));  // row_shr 1, 2, 4, 8
  v = max(v, dpp_or<0x112, 0xf>(INT32_MIN, v));
  v = max(v, dpp_or<0x114, 0xf>(INT32_MIN, v));
  v = max(v, dpp_or<0x118, 0xf>(INT32_MIN, v));
  v = max(v, dpp_or<0x142, 0xa>(INT32_MIN, v));  // row_bcast 15, 31
  v = max(v, dpp_or<0x143, 0xc>(INT32_MIN, v));
  return __builtin_amdgcn_readlane(v, 63);
}
// Sums of the lanes up to each one.
__device__ __forceinline__ int32_t wave_scan(int32_t v) {
  v += dpp_or<0x111, 0xf>(0, v);
  v += dpp_or<0x112, 0xf>(0, v);
  v += dpp_or<0x114, 0xf>(0, v);
  v += dpp_or<0x118, 0xf>(0, v);
  v += dpp_or<0x142, 0xa>(0, v);
  v += dpp_or<0x143, 0xc>(0, v);
  return v;
}
__device__ __forceinline__ uint32_t scalar_sum(uint32_t u) {
  return (uint32_t)__builtin_amdgcn_readlane(wave_scan((int32_t)u), 63);
}
// Of values below 2^36.
__device__ __forceinline__ uint64_t scalar_sum_u64(uint64_t v) {
  return ((uint64_t)scalar_sum((uint32_t)(v >> 20)) << 20) + scalar_sum((uint32_t)v & 0xfffffu);
}

__device__ __forceinline__ int32_t bit_length(uint64_t v) {
  return 64 - (v ? __clzll((long long)v) : 64);
}

}  // namespace ilw
