// grouped.hip -- int8 linear layers grouped by expert: rows sorted by expert,
// each expert its own weights, ragged numbers of rows.
//
//   y[m][n] = sat8(rq(b[e][n] + sum_k x[r(m)][k] w[e][n][k]; rq[e][n]))
//
// The grid holds as many tiles as any split of M rows over E experts can need
// (floor(M / TM) + E token tiles); a workgroup finds its expert from the offsets
// by a wave-wide scan over the experts' tile counts and leaves if there is none.
// A tile is WN x WM waves of FI x FJ MFMA tiles of 16 channels x 16 tokens.
// Operands go from memory straight to LDS, 16 bytes a lane, in two buffers: the
// loads of step k + 1 are in flight during the products of step k.
#include "ilw_internal.h"

namespace ilw {
namespace {

constexpr int NXCD = 8;

__device__ __forceinline__ int32_t wave_scan_i32(int32_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t t = __shfl_up(v, o, 64);
    v += lane >= o ? t : 0;
  }
  return v;
}

// Expert and rows m0 .. m1 - 1 (at most TM) of a token tile; m0 == m1: none.
struct Tile {
  int32_t e, m0, m1;
};
template <int TM>
__device__ __forceinline__ Tile find_tile(const GroupedArgs& a, int32_t tile, int lane) {
  int32_t before = 0;
  for (int32_t e0 = 0; e0 < a.E; e0 += 64) {
    const int32_t e = e0 + lane;
    int32_t lo = 0, hi = 0;
    if (e < a.E) {
      lo = min(max(a.offsets[e], 0), (int32_t)a.M);
      hi = min(max(a.offsets[e + 1], lo), (int32_t)a.M);
    }
    const int32_t n = (hi - lo + TM - 1) / TM, sum = before + wave_scan_i32(n, lane);
    const uint64_t hit = __ballot(sum > tile);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      const int32_t first = __shfl(sum - n, l, 64);
      const int32_t m0 = __shfl(lo, l, 64) + (tile - first) * TM, m1 = __shfl(hi, l, 64);
      return {__builtin_amdgcn_readfirstlane(e0 + l), __builtin_amdgcn_readfirstlane(m0),
              __builtin_amdgcn_readfirstlane(min(m0 + TM, m1))};
    }
    before = __shfl(sum, 63, 64);
  }
  return {0, 0, 0};
}

__device__ __forceinline__ void load_lds16(const int8_t* src, int8_t* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt 0

template <int WN, int WM, int FI, int FJ, int KB, bool KTAIL>
__global__ __launch_bounds__(64 * WN * WM) void grouped_kernel(GroupedArgs a, uint32_t tiles_n,
                                                              uint32_t tiles_total) {
  constexpr int WTN = 16 * FI, WTM = 16 * FJ, TN = WTN * WN, TM = WTM * WM, NW = WN * WM,
                NT = 64 * NW;
  constexpr int CPR = KB / 16, STAGE = (TN + TM) * KB;
  constexpr int OSTR = (TN / 4) % 8 == 0 ? TN / 4 + 4 : TN / 4;  // words per staged token row
  constexpr int SOUT = TM * OSTR * 4;
  __shared__ __attribute__((aligned(1024))) int8_t sbuf[2 * STAGE > SOUT ? 2 * STAGE : SOUT];
  __shared__ RqI64 rqc[TN];
  __shared__ int32_t unbounded;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const uint32_t bid = blockIdx.x;
  const uint32_t per = tiles_total / NXCD, rem = tiles_total % NXCD, xcd = bid % NXCD;
  const uint32_t t = xcd * per + min(xcd, rem) + bid / NXCD;
  const uint32_t tm = t / tiles_n;
  const int32_t n0 = (int32_t)(t - tm * tiles_n) * TN;
  const Tile tl = find_tile<TM>(a, (int32_t)tm, lane);
  if (tl.m0 >= tl.m1) return;
  const int32_t N = a.N, K = a.K;
  const int8_t* W = a.w + (int64_t)tl.e * N * K;

  // Each thread's 16-byte chunks of a step: LDS chunk id c = tid + i NT holds
  // chunk (c % CPR) ^ swizzle of row c / CPR (weights first, then tokens).
  constexpr int PT = (TN + TM) * CPR / NT;
  static_assert((TN + TM) * CPR % NT == 0 && TN * CPR % NT == 0, "whole rows a pass");
  const int8_t* src[PT];
  int kofs;
  {
    const int r = tid / CPR;  // rows of later chunks are r + i NT / CPR: the same swizzle
    static_assert((NT / CPR) % 8 == 0, "the swizzle repeats every 8 rows");
    kofs = ((tid % CPR) ^ (CPR == 8 ? (r & 6) : (r & 4) >> 1)) * 16;
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int row = r + i * (NT / CPR);
      if (row < TN) {
        src[i] = W + (int64_t)min(n0 + row, N - 1) * K;
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
  }
  const int nk = (K + KB - 1) / KB;
  auto load = [&](int kt, int buf) {
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
  };
  load(0, 0);
  bool clamp_acc = false;
  for (int c = tid; c < TN; c += NT) {
    const int64_t n = (int64_t)tl.e * N + min(n0 + c, N - 1), q = a.nq == 1 ? 0 : n;
    RqI64 r;
    clamp_acc |= !r.init_bounded(a.mult[q], a.shift[q], a.bias ? a.bias[n] : 0, (uint32_t)K << 14);
    rqc[c] = r;
  }
  if (tid == 0) unbounded = 0;
  const v4i zero = {0, 0, 0, 0};
  v4i acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = zero;
  int frag_off[KB / 64];
#pragma unroll
  for (int h = 0; h < KB / 64; ++h) frag_off[h] = lds_chunk<CPR>(lane & 15, h * 4 + (lane >> 4));
  auto compute = [&](int buf) {
    const int8_t* sw = sbuf + buf * STAGE + wn * WTN * KB;
    const int8_t* sx = sbuf + buf * STAGE + (TN + wm * WTM) * KB;
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
  };
  wait_loads();
  lds_sync();
  if (clamp_acc) unbounded = 1;  // (published by the loop's barriers)
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + 1 < nk) load(kt + 1, (kt + 1) & 1);
    compute(kt & 1);
    wait_loads();
    lds_sync();
  }

  // Epilogue: requantize, transpose through LDS, 16-byte row chunks out.
  bool dead[FJ];  // tokens whose row index points nowhere
#pragma unroll
  for (int j = 0; j < FJ; ++j) {
    dead[j] = false;
    if (a.rows) {
      const int32_t m = min(tl.m0 + wm * WTM + j * 16 + (lane & 15), tl.m1 - 1);
      dead[j] = (uint64_t)(int64_t)a.rows[m] >= (uint64_t)a.x_rows;
    }
  }
  uint32_t* so = (uint32_t*)sbuf;
  auto requant = [&](auto general) {
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int c = wn * WTN + i * 16 + (lane >> 4) * 4;
      RqI64 rf[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) rf[r] = rqc[c + r];
#pragma unroll
      for (int j = 0; j < FJ; ++j) {
        int32_t u[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int32_t v = dead[j] ? 0 : acc[i][j][r];
          u[r] = decltype(general)::value ? rf[r].apply(v) : rf[r].apply_unclamped(v);
        }
        so[(wm * WTM + j * 16 + (lane & 15)) * OSTR + (c >> 2)] = pack4(u[0], u[1], u[2], u[3]);
      }
    }
  };
  if (unbounded) requant(Flag<true>{});
  else requant(Flag<false>{});
  lds_sync();
  const bool a16 = ((uintptr_t)a.y & 15) == 0;
  for (int c = tid; c < TM * (TN / 16); c += NT) {
    const int r = c / (TN / 16), q = c - r * (TN / 16);
    const int32_t n = n0 + q * 16;
    if (tl.m0 + r >= tl.m1 || n >= N) continue;
    int8_t* dst = a.y + (int64_t)(tl.m0 + r) * N + n;
    const v4i v = *(const v4i*)(so + r * OSTR + q * 4);
    if (a16) {
      *(v4i*)dst = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) ((int32_t*)dst)[i] = v[i];
    }
  }
}

template <int WN, int WM, int FI, int FJ, int KB>
hipError_t launch_cfg(const GroupedArgs& a, hipStream_t s) {
  constexpr int TN = 16 * FI * WN, TM = 16 * FJ * WM;
  const uint32_t tiles_n = (uint32_t)((a.N + TN - 1) / TN);
  const int64_t tiles_m = a.M / TM + (a.E < a.M ? a.E : a.M), total = tiles_m * tiles_n;
  if (total * 64 * WN * WM >= ((int64_t)1 << 32)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)total), block(64 * WN * WM);
  if (a.K % KB == 0)
    hipLaunchKernelGGL((grouped_kernel<WN, WM, FI, FJ, KB, false>), grid, block, 0, s, a, tiles_n,
                       (uint32_t)total);
  else
    hipLaunchKernelGGL((grouped_kernel<WN, WM, FI, FJ, KB, true>), grid, block, 0, s, a, tiles_n,
                       (uint32_t)total);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped(const GroupedArgs& a, hipStream_t s) {
  return launch_cfg<2, 2, 4, 4, 128>(a, s);
}

}  // namespace ilw
