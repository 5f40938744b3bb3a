// expert_tiles.h -- tiles of an int8 product over rows that may be sorted by
// expert, shared by the linears grouped by expert and those with token and channel
// scales: which expert, rows and channels a workgroup has, and the sums of its tile.
//
// The grid holds as many tiles as any split of M rows over E experts can need
// (floor(M / TM) + E token tiles); a workgroup finds its expert from the offsets
// by a wave-wide scan over the experts' tile counts and leaves if there is none.
// A tile is WN x WM waves of FI x FJ MFMA tiles of 16 channels x 16 tokens.
// Operands go from memory straight to LDS, 16 bytes a lane, in S buffers: the loads of
// the next S - 1 steps are in flight during the products of a step.  (Weights read
// straight to registers where few rows use them: 34 us against 22, since a load
// then takes 64 bytes of 16 rows where these take whole 128-byte lines.)
#pragma once
#include "ilw_internal.h"

namespace ilw {
constexpr int NXCD = 8;
constexpr int KB = 128;  // inputs of a step: one cache line of each row

__device__ __forceinline__ int32_t wave_scan_i32(int32_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t t = __shfl_up(v, o, 64);
    v += lane >= o ? t : 0;
  }
  return v;
}

// A workgroup's tile: expert e, rows m0 .. m1 - 1 (at most TM; m0 == m1: none),
// channels from n0 on.
struct Tile {
  int32_t e, m0, m1, n0;
};
// The tiles that hold rows are numbered expert by expert, the channel tiles of a
// token tile next to each other, and each XCD takes one run of numbers: what
// shares rows or weights shares an L2. The run is a share of the tiles there are,
// not of the grid, whose last tiles are the ones that the offsets leave without rows.
template <int TM, int TN, typename Args>
__device__ __forceinline__ Tile find_tile(const Args& a, uint32_t tiles_n, int lane) {
  const auto count = [&](int32_t e, int32_t& lo, int32_t& hi) {
    lo = hi = 0;
    if (!a.offsets) {  // every row is of the one expert
      hi = e == 0 ? (int32_t)a.M : 0;
    } else if (e < a.E) {
      lo = min(max(a.offsets[e], 0), (int32_t)a.M);
      hi = min(max(a.offsets[e + 1], lo), (int32_t)a.M);
    }
    return (hi - lo + TM - 1) / TM;
  };
  int32_t lo, hi, n = count(lane, lo, hi), sum = wave_scan_i32(n, lane);
  uint32_t live = __builtin_amdgcn_readlane(sum, 63);
  for (int32_t e0 = 64; e0 < a.E; e0 += 64) {
    int32_t l, h;
    live += __builtin_amdgcn_readlane(wave_scan_i32(count(e0 + lane, l, h), lane), 63);
  }
  live *= tiles_n;
  const uint32_t xcd = blockIdx.x % NXCD, i = blockIdx.x / NXCD, per = live / NXCD,
                 rem = live % NXCD;
  if (i >= per + (xcd < rem)) return {0, 0, 0, 0};
  const uint32_t t = xcd * per + min(xcd, rem) + i, tm = t / tiles_n;
  const int32_t tile = (int32_t)tm, n0 = (int32_t)(t - tm * tiles_n) * TN;
  for (int32_t e0 = 0;;) {
    const uint64_t hit = __ballot(sum > tile);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      const int32_t m0 = __builtin_amdgcn_readlane(lo, l) +
                         (tile - __builtin_amdgcn_readlane(sum - n, l)) * TM;
      return {e0 + l, m0, min(m0 + TM, __builtin_amdgcn_readlane(hi, l)), n0};
    }
    e0 += 64;
    if (e0 >= a.E) return {0, 0, 0, 0};
    const int32_t before = __builtin_amdgcn_readlane(sum, 63);
    n = count(e0 + lane, lo, hi);
    sum = before + wave_scan_i32(n, lane);
  }
}

__device__ __forceinline__ void load_lds16(const int8_t* src, int8_t* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

template <int N = 0>
__device__ __forceinline__ void wait_loads() {  // all but the last N vector loads
  static_assert(N < 64, "the counter's range");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

// The sums of a tile. Args has x, rows (or null), w, x_rows, N, K; the LDS buffer
// holds S STAGE bytes, 1024-byte aligned: S - 1 steps are loaded ahead.
template <int WN, int WM, int FI, int FJ, bool KTAIL, int S = 2>
struct TileProduct {
  static constexpr int WTN = 16 * FI, WTM = 16 * FJ, TN = WTN * WN, TM = WTM * WM,
                       NT = 64 * WN * WM;
  static constexpr int CPR = KB / 16, STAGE = (TN + TM) * KB;
  // Each thread's 16-byte chunks of a step: LDS chunk id c = tid + i NT holds
  // chunk (c % CPR) ^ swizzle of row c / CPR (weights first, then tokens).
  static constexpr int PT = (TN + TM) * CPR / NT;
  static_assert((TN + TM) * CPR % NT == 0 && TN * CPR % NT == 0, "whole rows a pass");
  static_assert((NT / CPR) % 8 == 0, "the swizzle repeats every 8 rows");
  const int8_t* src[PT];
  int32_t kofs, K;
  int lane, wave;
  int8_t* sbuf;
  v4i acc[FI][FJ];

  // The addresses, and the first steps' loads.
  template <typename Args>
  __device__ __forceinline__ void start(const Args& a, const Tile& tl, int8_t* lds, int tid) {
    K = a.K;
    lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    sbuf = lds;
    const int8_t* W = a.w + (int64_t)tl.e * a.N * K;
    const int r = tid / CPR;  // rows of later chunks are r + i NT / CPR: the same swizzle
    kofs = ((tid % CPR) ^ (r & 6)) * 16;
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int row = r + i * (NT / CPR);
      if (row < TN) {
        src[i] = W + (int64_t)min(tl.n0 + row, a.N - 1) * K;
      } else {
        const int32_t m = min(tl.m0 + row - TN, tl.m1 - 1);
        int64_t xr = m;
        if (a.rows) {
          xr = a.rows[m];
          xr = (uint64_t)xr < (uint64_t)a.x_rows ? xr : 0;  // (zeroed in the epilogue)
        }
        src[i] = a.x + xr * K;
      }
    }
#pragma unroll
    for (int i = 0; i + 1 < S; ++i)
      if (i == 0 || i * KB < K) load(i, i);
  }
  __device__ __forceinline__ void load(int kt, int buf) {
    int8_t* dst = sbuf + buf * STAGE + wave * 1024;
    const int k = kt * KB + kofs;
    if (!KTAIL || kt * KB + KB <= K) {
#pragma unroll
      for (int i = 0; i < PT; ++i) load_lds16(src[i] + k, dst + i * (NT * 16));
    } else {
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        v4i v = {0, 0, 0, 0};
        if (k < K) v = *(const v4i*)(src[i] + k);
        *(v4i*)(dst + i * (NT * 16) + lane * 16) = v;
      }
    }
  }
  // The first steps' loads have arrived (and what the workgroup wrote to LDS).
  __device__ __forceinline__ void ready() {
    wait_loads();
    lds_sync();
  }
  __device__ __forceinline__ void run() {
    const int wn = wave % WN, wm = wave / WN, nk = (K + KB - 1) / KB;
    const v4i zero = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = zero;
    int frag_off[KB / 64];
#pragma unroll
    for (int h = 0; h < KB / 64; ++h) frag_off[h] = lds_chunk<CPR>(lane & 15, h * 4 + (lane >> 4));
    int ring = 0;
    for (int kt = 0; kt < nk; ++kt) {
      const int ahead = kt + S - 1, buf = S == 2 ? kt & 1 : ring;
      if (ahead < nk) load(ahead, S == 2 ? ahead & 1 : buf == 0 ? S - 1 : buf - 1);
      const int8_t* sw = sbuf + buf * STAGE + wn * WTN * KB;
      const int8_t* sx = sbuf + buf * STAGE + (TN + wm * WTM) * KB;
      ring = ring + 1 == S ? 0 : ring + 1;
#pragma unroll
      for (int h = 0; h < KB / 64; ++h) {
        v4i fa[FI], fb[FJ];
#pragma unroll
        for (int i = 0; i < FI; ++i) fa[i] = *(const v4i*)(sw + i * 16 * KB + frag_off[h]);
#pragma unroll
        for (int j = 0; j < FJ; ++j) fb[j] = *(const v4i*)(sx + j * 16 * KB + frag_off[h]);
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
          for (int j = 0; j < FJ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
      }
      // (the last steps, and one that is not loaded straight to LDS, count as none)
      if (S > 2 && ahead < nk - KTAIL) wait_loads<(S - 2) * PT>();
      else wait_loads();
      lds_sync();
    }
  }
};

}  // namespace ilw
