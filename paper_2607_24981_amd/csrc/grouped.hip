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
// loads of step k + 1 are in flight during the products of step k.  (Weights read
// straight to registers where few rows use them: 34 us against 22, since a load
// then takes 64 bytes of 16 rows where these take whole 128-byte lines.)
#include "decoder_internal.h"

namespace ilw {
namespace {

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
template <int TM, int TN>
__device__ __forceinline__ Tile find_tile(const GroupedArgs& a, uint32_t tiles_n, int lane) {
  const auto count = [&](int32_t e, int32_t& lo, int32_t& hi) {
    lo = hi = 0;
    if (e < a.E) {
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

__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt 0

template <int WN, int WM, int FI, int FJ, bool KTAIL>
__global__ __launch_bounds__(64 * WN * WM) void grouped_kernel(GroupedArgs a, uint32_t tiles_n) {
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
  const Tile tl = find_tile<TM, TN>(a, tiles_n, lane);
  if (tl.m0 >= tl.m1) return;
  const int32_t N = a.N, K = a.K, n0 = tl.n0;
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
    kofs = ((tid % CPR) ^ (r & 6)) * 16;
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

template <int WN, int WM, int FI, int FJ>
hipError_t launch_cfg(const GroupedArgs& a, hipStream_t s) {
  constexpr int TN = 16 * FI * WN, TM = 16 * FJ * WM;
  const uint32_t tiles_n = (uint32_t)((a.N + TN - 1) / TN);
  const int64_t tiles_m = a.M / TM + (a.E < a.M ? a.E : a.M), total = tiles_m * tiles_n;
  // total * block < 2^32: the entry point holds (M / 64 + E) (N / 128 + 1) below 2^22,
  // and the one tile of 1024 threads has E <= M / 192
  const dim3 grid((unsigned)total), block(64 * WN * WM);
  if (a.K % KB == 0)
    hipLaunchKernelGGL((grouped_kernel<WN, WM, FI, FJ, false>), grid, block, 0, s, a, tiles_n);
  else
    hipLaunchKernelGGL((grouped_kernel<WN, WM, FI, FJ, true>), grid, block, 0, s, a, tiles_n);
  return hipGetLastError();
}

}  // namespace

// Which tile, by M / E rows an expert and by S = M N / 65536, about the number of
// 256 x 256 tiles; the offsets are on the device, so what an expert really has is
// not known here.  Times in us at uniformly random experts, int8:
//   256 x 256, 16 waves (4 a SIMD hide what 1 or 2 cannot: 400 us at 49152 rows of
//     32 experts, N 2048, K 4096, 2060 Tops; the same tile of 8 waves 405, 128 x 128
//     of 8 waves 465, of 4 waves 485).  M 12288, E 64, N 4096, K 4096: 270, next 320.
//     At 96 rows an expert half of it is empty: 250 against 202; with S 96 it
//     leaves CUs idle: 55 against 40.
//   128 x 128, 8 waves: M 1536, E 8, N 4096, K 4096: 40 against 58 of 64 rows; with
//     S 12 it is as good as these, 12.2 against 12.1.
//   256 channels x 32 rows: weights come in once, at 6.0 TB/s where 64 experts are
//     2048 x 1024 and have 4 rows each (22 us; 64 rows 26, 128 x 128 27), if two
//     workgroups a CU can be had: at 8 experts of 4096 x 4096 38 against 34.
//   128 channels x 64 rows: everything between.
hipError_t launch_grouped(const GroupedArgs& a, hipStream_t s) {
  const int64_t size = a.M * a.N, unit = 65536;
  if (a.M >= 192 * (int64_t)a.E && size > 128 * unit) return launch_cfg<4, 4, 4, 4>(a, s);
  if (a.M >= 64 * (int64_t)a.E && size >= 24 * unit) return launch_cfg<2, 4, 4, 2>(a, s);
  if (a.M <= 16 * (int64_t)a.E && a.E * (int64_t)((a.N + 255) / 256) >= 512)
    return launch_cfg<4, 1, 4, 2>(a, s);
  return launch_cfg<2, 2, 4, 2>(a, s);
}

}  // namespace ilw
