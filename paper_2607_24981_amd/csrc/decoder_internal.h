// decoder_internal.h -- arguments and launchers of the paged cache and the linears
// grouped by expert.
#pragma once
#include "ilw_internal.h"

namespace ilw {

// Paged int8 cache (see ilw_kv_cache), page size 1 << lp.
struct CacheView {
  int8_t* k;
  int8_t* v;
  int32_t* k_scale;
  int32_t* v_scale;
  const int32_t* table;
  int32_t n_pages, max_pages, Hkv, D, lp;
};
struct AppendArgs {
  CacheView c;
  const int8_t* qkv;
  int64_t ld;
  const int32_t* cu;
  const int32_t* past;
  const int16_t* rope;
  int32_t R, inter;
  int8_t* q;
  int32_t* q_scale;
  int32_t T, seqs, max_new, Hq;
};
bool cache_append_fits(const AppendArgs& a);  // one launch can hold it
hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s);

struct CacheAttnArgs {
  CacheView c;
  const int8_t* q;
  const int32_t* q_scale;
  const int32_t* cu;
  const int32_t* lens;
  int8_t* out;
  int32_t T, seqs, max_q, max_len, Hq;
  int32_t score_mult, score_t, out_mult, out_shift, causal, window;
  int32_t out_clamp;  // set by launch_cache_attention
};
bool cache_attention_fits(const CacheAttnArgs& a);  // its launches can hold it
size_t cache_attention_workspace(const CacheAttnArgs& a);
hipError_t launch_cache_attention(const CacheAttnArgs& a, void* ws, hipStream_t s);

// Linear layers grouped by expert (see ilw_linear_grouped).
struct GroupedArgs {
  const int8_t* x;
  const int32_t* rows;     // or null
  const int32_t* offsets;  // [E + 1]
  const int8_t* w;
  const int32_t* bias;     // or null
  const int32_t* mult;
  const int32_t* shift;
  int8_t* y;
  int64_t M, x_rows;
  int32_t nq, E, N, K;
};
hipError_t launch_grouped(const GroupedArgs& a, hipStream_t s);

}  // namespace ilw
