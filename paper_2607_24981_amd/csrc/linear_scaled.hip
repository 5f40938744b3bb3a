// linear_scaled.hip -- int8 products with a scale for each token and a factor for
// each channel, dense or grouped by expert, int16 or int8 out.
//
//   y[m][n] = sat(floor((floor(acc F / 2^max(q - 4, 0)) + b + 8) / 16))
// F = floor(X Y / 2^32) of the token's scale X = S 2^z in [2^31, 2^32) and the
// channel's multiplier Y = mult 2^u in [2^30, 2^31), so that F is in [2^29, 2^31)
// and keeps 29 bits or more whatever the scales are; q = shift + z + u - 18.  A sum of
// K products is below 2^14 K, so with e bits to spare, floor(acc F / 2^(q - 4)) is the
// high word of (acc 2^e) F shifted right by q - 36 + e, from q = 36 - e on: two 32-bit
// high products, two adds, three shifts and a median a value.  (q of a layer whose
// outputs use their bits is 30 + the sums' bits - the outputs'.)  Below that the
// 64-bit product is shifted.
//
// Tiles and their sums: expert_tiles.h.
#include "step_internal.h"
#include "expert_tiles.h"

namespace ilw {
namespace {

struct Channel {
  uint32_t Y;
  int32_t q;  // shift + u - 22: q - 4 without the token's z
  int32_t c;  // b + 8
};
__device__ __forceinline__ Channel channel_of(int32_t mult, int32_t shift, int32_t b) {
  Channel r;
  const int32_t u = mult > 0 ? __clz(mult) - 1 : 0;
  r.Y = mult > 0 ? (uint32_t)mult << u : 0;
  r.q = mult > 0 ? shift + u - 22 : 64;  // (64: no factor, no bound on anything)
  r.c = min(max(b, -(1 << 24)), 1 << 24) + 8;
  return r;
}
struct Token {
  uint32_t X;
  int32_t z;
};
__device__ __forceinline__ Token token_of(int32_t S) {
  Token r;
  r.z = S > 0 ? __clz(S) : 31;
  r.X = S > 0 ? (uint32_t)S << r.z : 0;
  return r;
}
// Bits that a sum of K products leaves free.
__device__ __forceinline__ int32_t spare_bits(int32_t K) { return max(__clz(K) - 15, 0); }
// One output before saturation; FAST: q >= 36 - e, e the sums' spare bits.
template <bool FAST>
__device__ __forceinline__ int32_t scaled(int32_t acc, const Channel& c, const Token& t, int32_t e) {
  const int32_t F = (int32_t)__umulhi(t.X, c.Y);
  const int32_t s = c.q + t.z;
  if (FAST) return ((__mulhi((int32_t)((uint32_t)acc << e), F) >> min(s - 32 + e, 31)) + c.c) >> 4;
  const int64_t v = (((int64_t)acc * F) >> min(max(s, 0), 63)) + c.c;
  return (int32_t)min(max(v >> 4, (int64_t)-65536), (int64_t)65536);
}

template <int WN, int WM, int FI, int FJ, int BYTES, bool KTAIL, int S>
__global__ __launch_bounds__(64 * WN * WM) void scaled_kernel(ScaledArgs a, uint32_t tiles_n) {
  using Product = TileProduct<WN, WM, FI, FJ, KTAIL, S>;
  constexpr int WTN = Product::WTN, WTM = Product::WTM, TN = Product::TN, TM = Product::TM,
                NT = Product::NT, STAGE = Product::STAGE;
  constexpr int OSTR = TN * BYTES / 4 + 4;  // words per staged token row
  constexpr int SOUT = TM * OSTR * 4;
  __shared__ __attribute__((aligned(1024))) int8_t sbuf[S * STAGE > SOUT ? S * STAGE : SOUT];
  __shared__ Channel chan[TN];
  __shared__ Token token[TM];
  __shared__ int32_t least_q, least_z;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const Tile tl = find_tile<TM, TN>(a, tiles_n, lane);
  if (tl.m0 >= tl.m1) return;
  const int32_t N = a.N, n0 = tl.n0;
  Product p;
  p.start(a, tl, sbuf, tid);
  int32_t q = INT32_MAX;
  for (int c = tid; c < TN; c += NT) {
    const int64_t n = (int64_t)tl.e * N + min(n0 + c, N - 1), r = a.nq == 1 ? 0 : n;
    const Channel ch = channel_of(a.mult[r], a.shift[r], a.bias ? a.bias[n] : 0);
    chan[c] = ch;
    q = min(q, ch.q);
  }
  int32_t z = 31;
  for (int t = tid; t < TM; t += NT) {
    const int32_t m = min(tl.m0 + t, tl.m1 - 1);
    int64_t r = m;
    if (a.rows) r = a.rows[m];
    // a row index that points nowhere is a row of zeros: no factor at all
    const Token tk = token_of((uint64_t)r < (uint64_t)a.x_rows ? a.x_scale[r] : 0);
    token[t] = tk;
    z = min(z, tk.z);
  }
  if (tid == 0) least_q = INT32_MAX, least_z = 31;
  p.ready();
  atomicMin(&least_q, q);  // (published by the loop's barriers)
  atomicMin(&least_z, z);
  p.run();

  // Epilogue: scale, transpose through LDS, 16-byte row chunks out.
  const int32_t spare = spare_bits(a.K);
  uint32_t* so = (uint32_t*)sbuf;
  auto scale = [&](auto fast) {
    constexpr int32_t lim = BYTES == 1 ? 127 : 32767;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int c = wn * WTN + i * 16 + (lane >> 4) * 4;
      Channel ch[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) ch[r] = chan[c + r];
#pragma unroll
      for (int j = 0; j < FJ; ++j) {
        __builtin_amdgcn_sched_barrier(0);  // (four values at a time: more would spill)
        const Token tok = token[wm * WTM + j * 16 + (lane & 15)];
        int32_t v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          v[r] = min(max(scaled<decltype(fast)::value>(p.acc[i][j][r], ch[r], tok, spare), -lim), lim);
        uint32_t* dst = so + (wm * WTM + j * 16 + (lane & 15)) * OSTR + (c * BYTES >> 2);
        if (BYTES == 1) {
          *dst = pack4(v[0], v[1], v[2], v[3]);
        } else {
          dst[0] = __builtin_amdgcn_perm((uint32_t)v[1], (uint32_t)v[0], 0x05040100u);
          dst[1] = __builtin_amdgcn_perm((uint32_t)v[3], (uint32_t)v[2], 0x05040100u);
        }
      }
    }
  };
  if (least_q + least_z >= 32 - spare) scale(Flag<true>{});
  else scale(Flag<false>{});
  lds_sync();
  constexpr int CH = TN * BYTES / 16;  // 16-byte chunks of a row
  const bool a16 = ((uintptr_t)a.y & 15) == 0;
  for (int c = tid; c < TM * CH; c += NT) {
    const int r = c / CH, k = c - r * CH;
    const int32_t n = n0 + k * (16 / BYTES);
    if (tl.m0 + r >= tl.m1 || n >= N) continue;
    int8_t* dst = (int8_t*)a.y + ((int64_t)(tl.m0 + r) * N + n) * BYTES;
    const v4i v = *(const v4i*)(so + r * OSTR + k * 4);
    if (a16) {
      *(v4i*)dst = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) ((int32_t*)dst)[i] = v[i];
    }
  }
}

// Few rows: the weights are what takes time.  A workgroup has 16 FI channels and 16 FJ
// rows, its waves share K in steps of 128 (wave w: steps w, w + NW, ...), and each
// wave streams its own weights through a ring of R steps in LDS that no other wave
// touches, so no barrier holds the loads back; the rows come straight to registers.
// The waves' sums meet in LDS at the end.
template <int N>
__device__ __forceinline__ void wait_vm() {  // all but the last N vector loads
  static_assert(N < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
// A step's weights out of a slot, at LDS addresses a (first 64 inputs) and b, 16
// channels each 2 KB; they are in the registers when it is done, so the slot may be
// loaded again.  (Written as ordinary reads, the first slot's wait for the loads of
// all slots: the compiler does not tell what lies between them.)
template <int FI>
__device__ __forceinline__ void read_step(v4i (&w)[2][FI], int a, int b) {
  static_assert(FI == 1 || FI == 2 || FI == 4, "the reads below");
  if constexpr (FI == 1)
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(w[0][0]), "=&v"(w[1][0])
                 : "v"(a), "v"(b)
                 : "memory");
  else if constexpr (FI == 2)
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:2048\n\t"
        "ds_read_b128 %2, %5\n\tds_read_b128 %3, %5 offset:2048\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[1][0]), "=&v"(w[1][1])
        : "v"(a), "v"(b)
        : "memory");
  else
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:2048\n\t"
        "ds_read_b128 %2, %8 offset:4096\n\tds_read_b128 %3, %8 offset:6144\n\t"
        "ds_read_b128 %4, %9\n\tds_read_b128 %5, %9 offset:2048\n\t"
        "ds_read_b128 %6, %9 offset:4096\n\tds_read_b128 %7, %9 offset:6144\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(w[0][0]), "=&v"(w[0][1]), "=&v"(w[0][2]), "=&v"(w[0][3]), "=&v"(w[1][0]),
          "=&v"(w[1][1]), "=&v"(w[1][2]), "=&v"(w[1][3])
        : "v"(a), "v"(b)
        : "memory");
}

template <int R, typename F>
__device__ __forceinline__ void steps_of(F f) {
  static_assert(R == 2 || R == 4, "the steps below");
  f(IntC<0>{});
  f(IntC<1>{});
  if constexpr (R == 4) {
    f(IntC<2>{});
    f(IntC<3>{});
  }
}

typedef uint32_t u32x2a4 __attribute__((ext_vector_type(2), aligned(4)));

template <int FI, int FJ, int NW, int R, int BYTES>
__global__ __launch_bounds__(64 * NW) void stream_kernel(ScaledArgs a, uint32_t tiles_n) {
  constexpr int TN = 16 * FI, TM = 16 * FJ, NT = 64 * NW, STEP = TN * KB, RING = R * STEP;
  constexpr int WL = 2 * FI, XL = 2 * FJ;  // loads of a step: weights, rows
  static_assert(FI * FJ * 1024 <= RING, "a wave's sums fit its ring");
  static_assert(TN <= NT && TM <= NT, "a thread a constant");
  __shared__ __attribute__((aligned(1024))) int8_t ring[NW * RING];
  __shared__ Channel chan[TN];
  __shared__ Token token[TM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Tile tl = find_tile<TM, TN>(a, tiles_n, lane);
  if (tl.m0 >= tl.m1) return;
  const int32_t N = a.N, K = a.K, n0 = tl.n0;

  // Row numbers, scales and constants first: loads return in order, and from the
  // weights on a wait is for the step that it is meant for.  Scales and constants stay
  // in registers until the sums are there.
  int32_t xr[FJ], tr = min(tl.m0 + min(tid, TM - 1), tl.m1 - 1);
#pragma unroll
  for (int j = 0; j < FJ; ++j) xr[j] = min(tl.m0 + j * 16 + (lane & 15), tl.m1 - 1);
  if (a.rows) {
    tr = a.rows[tr];
#pragma unroll
    for (int j = 0; j < FJ; ++j) xr[j] = a.rows[xr[j]];
  }
  const bool there = (uint64_t)(int64_t)tr < (uint64_t)a.x_rows;
  tr = there ? tr : 0;
  const int8_t* xp[FJ];
#pragma unroll
  for (int j = 0; j < FJ; ++j)
    xp[j] = a.x + ((uint64_t)(int64_t)xr[j] < (uint64_t)a.x_rows ? (int64_t)xr[j] : 0) * K;
  const int32_t S = a.x_scale[tr];
  const int64_t cn = (int64_t)tl.e * N + min(n0 + min(tid, TN - 1), N - 1);
  const int32_t mult = a.mult[a.nq == 1 ? 0 : cn], shift = a.shift[a.nq == 1 ? 0 : cn];
  const int32_t some = (a.bias ? a.bias : a.mult)[a.bias ? cn : 0], bias = a.bias ? some : 0;

  // weights: load i has rows 8 i + lane / 8, chunk lane % 8 of the swizzled line
  const int8_t* wbase = a.w + ((int64_t)tl.e * N + n0) * K;
  const uint32_t wrow = (uint32_t)(lane >> 3) * (uint32_t)K, 
                 wend = (uint32_t)min(N - 1 - n0, TN - 1) * (uint32_t)K;  // the last row's
  const int32_t wk = ((lane & 7) ^ ((lane >> 3) & 6)) * 16;
  int8_t* mine = ring + wave * RING;
  const int32_t nk = (K + KB - 1) / KB, ns = nk > wave ? (nk - wave - 1) / NW + 1 : 0;
  // Workgroups begin at different steps: where rows are a power of two of bytes apart,
  // the same step of all of them would be in few memory channels.
  const int32_t turn = K % KB == 0 ? (n0 / TN) % nk : 0;
  const auto start_of = [&](int32_t s) {  // of the wave's step s
    const int32_t k = wave + s * NW + turn;
    return (k < nk ? k : k - nk) * KB;
  };
  const auto load_w = [&](int32_t s, int slot) {
    // (past the row's end: any of its bytes, the rows' zeros meet them)
    const uint32_t k = (uint32_t)min(start_of(s) + wk, K - 16);
#pragma unroll
    for (int i = 0; i < WL; ++i)
      load_lds16(wbase + (min(wrow + (uint32_t)(8 * i) * (uint32_t)K, wend) + k),
                 mine + slot * STEP + i * 1024);
  };
  v4i x[R][FJ][2];
  const int32_t xk = (lane >> 4) * 16;
  const auto load_x = [&](int32_t s, v4i (&v)[FJ][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t k = min(start_of(s) + h * 64 + xk, K - 16);
#pragma unroll
      for (int j = 0; j < FJ; ++j) v[j][h] = *(const v4i*)(xp[j] + k);
    }
  };
#pragma unroll
  for (int r = 0; r < R; ++r) {
    load_w(r, r);
    load_x(r, x[r]);
  }

  const v4i zero = {0, 0, 0, 0};
  v4i acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = zero;
  int frag[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    frag[h] = (int)(uintptr_t)(__attribute__((address_space(3))) int8_t*)mine +
              lds_chunk<8>(lane & 15, h * 4 + (lane >> 4));
  }
  const auto compute = [&](int slot, v4i (&v)[FJ][2]) {
    v4i w[2][FI];
    read_step<FI>(w, frag[0] + slot * STEP, frag[1] + slot * STEP);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[h][i], v[j][h], acc[i][j], 0, 0, 0);
  };
  // Rounds of R steps without a branch.  All but the last load the next round's steps
  // (which may lie past the end of the row: see load_w).
  const int32_t rounds = max((ns + R - 1) / R, 1);
  for (int32_t g = 0; g + 1 < rounds; ++g)
    steps_of<R>([&](auto slot) {
      constexpr int r = decltype(slot)::value;
      wait_vm<(R - 1) * (WL + XL)>();
      compute(r, x[r]);
      load_w((g + 1) * R + r, r);
      load_x((g + 1) * R + r, x[r]);
    });
  steps_of<R>([&](auto slot) {
    constexpr int r = decltype(slot)::value;
    const int32_t left = K - (wave + ((rounds - 1) * R + r) * NW) * KB;  // inputs from here on
    wait_vm<(R - 1 - r) * (WL + XL)>();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < FJ; ++j) x[r][j][h] = h * 64 + xk < left ? x[r][j][h] : zero;
    compute(r, x[r]);
  });

  // every wave's sums, each 16 x 16 tile 1 KB in the wave's ring
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) *(v4i*)(mine + (i * FJ + j) * 1024 + lane * 16) = acc[i][j];
  if (tid < TN) chan[tid] = channel_of(mult, shift, bias);
  // a row index that points nowhere is a row of zeros: no factor at all
  if (tid < TM) token[tid] = token_of(there ? S : 0);
  __syncthreads();
  constexpr int32_t lim = BYTES == 1 ? 127 : 32767;
  for (int f = wave; f < FI * FJ; f += NW) {
    const int i = f / FJ, j = f % FJ;
    v4i sum = zero;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += *(const v4i*)(ring + w * RING + f * 1024 + lane * 16);
    const int32_t t = j * 16 + (lane & 15), c = i * 16 + (lane >> 4) * 4;
    const Token tk = token[t];
    int32_t v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
      v[r] = min(max(scaled<false>(sum[r], chan[c + r], tk, 0), -lim), lim);
    if (tl.m0 + t >= tl.m1 || n0 + c >= N) continue;
    int8_t* dst = (int8_t*)a.y + ((int64_t)(tl.m0 + t) * N + n0 + c) * BYTES;
    if (BYTES == 1)
      *(uint32_t*)dst = pack4(v[0], v[1], v[2], v[3]);
    else
      *(u32x2a4*)dst = u32x2a4{__builtin_amdgcn_perm((uint32_t)v[1], (uint32_t)v[0], 0x05040100u),
                               __builtin_amdgcn_perm((uint32_t)v[3], (uint32_t)v[2], 0x05040100u)};
  }
}

template <int FI, int FJ, int NW, int R, int BYTES>
hipError_t launch_stream(const ScaledArgs& a, hipStream_t s) {
  constexpr int TN = 16 * FI, TM = 16 * FJ;
  const uint32_t tiles_n = (uint32_t)((a.N + TN - 1) / TN);
  const int64_t tiles_m =
      a.offsets ? a.M / TM + (a.E < a.M ? a.E : a.M) : (a.M + TM - 1) / TM;
  hipLaunchKernelGGL((stream_kernel<FI, FJ, NW, R, BYTES>), dim3((unsigned)(tiles_m * tiles_n)),
                     dim3(64 * NW), 0, s, a, tiles_n);
  return hipGetLastError();
}

template <int WN, int WM, int FI, int FJ, int BYTES, int S>
hipError_t launch_cfg(const ScaledArgs& a, hipStream_t s) {
  constexpr int TN = 16 * FI * WN, TM = 16 * FJ * WM;
  const uint32_t tiles_n = (uint32_t)((a.N + TN - 1) / TN);
  const int64_t tiles_m =
      a.offsets ? a.M / TM + (a.E < a.M ? a.E : a.M) : (a.M + TM - 1) / TM;
  // below 2^32 threads: the entry point holds (M / 64 + E) (N / 128 + 1) below 2^22,
  // and the one tile of 1024 threads has E <= M / 192
  const dim3 grid((unsigned)(tiles_m * tiles_n)), block(64 * WN * WM);
  if (a.K % KB == 0)
    hipLaunchKernelGGL((scaled_kernel<WN, WM, FI, FJ, BYTES, false, S>), grid, block, 0, s, a, tiles_n);
  else
    hipLaunchKernelGGL((scaled_kernel<WN, WM, FI, FJ, BYTES, true, S>), grid, block, 0, s, a, tiles_n);
  return hipGetLastError();
}

// Which kernel, by the rows an expert has on average (what it really has is on the
// device) and by how many workgroups c(TN, TM) = token tiles x channel tiles there
// are.  Times in us, weights from memory, N x K:
//   16 rows: up to 16 rows an expert, or as long as 32 channels a workgroup are at
//     most 256 workgroups (32 rows of 4096 x 2048: 5.5, 32-row tiles 5.9; 64 rows:
//     7.9 against 6.3).  64 channels from 1024 workgroups on (512 rows of 64 experts,
//     2048 x 1024: 28.4, 32 channels 30.0; 16 rows of 16384 x 2048: 8.5 against
//     8.2).  Few long rows take 16 channels and eight waves (1 row of 512 x 8192: 4.9
//     against 6.7; of 1024 x 1024: 3.8 against 3.4).
//   32 rows: up to 32 rows an expert, or up to 256 workgroups of 64 channels (512
//     rows of 1024 x 1024: 6.2, 64-row tiles 7.7; 256 rows of 4096 x 2048: 13.8
//     against 11.3).  32 channels up to 256 workgroups of them (64 rows of 4096 x
//     2048: 6.3, 64 channels 7.5).
//   64 rows: up to 64 rows an expert, or up to 512 workgroups (2048 rows of 1024 x
//     1024: 10.6, tiles of 128 x 128 13.5; 1024 rows of 4096 x 2048: 27.5 against 20.9).
//     Two waves from 1024 workgroups on (4096 rows of 64 experts, 2048 x 1024: 47.3, four
//     51.8; 64 rows of 32768 x 4096: 37.4 against 36.5).
//   More: tiles as of the linears grouped by expert, whose launch has both sides.  Up to
//     256 of 128 x 128, one a CU, load three steps ahead (4096 rows of 1024 x 8192: 48.4,
//     one step 66; 700 rows of 4096 x 4096: 26.8 and 29.8); more of them load one, so
//     that a CU has two (2048 rows of 4096 x 4096: 44.6, three steps 59.6).
// An expert with many more rows than the average has its weights read again, from L2, for
// each tile of them (512 rows of 64 experts, 503 of them one's, 2048 x 1024: 11.0, 512
// rows of one expert in its own tiles 8.8).
template <int BYTES>
hipError_t launch_bytes(const ScaledArgs& a, hipStream_t s) {
  // (every grid below 2^32 threads: the entry point holds (M / 64 + E) (N / 128 + 1)
  // below 2^22, and the streams that are not limited here have M <= 64 E)
  const int64_t E = a.E, size = a.M * a.N, unit = 65536;
  const auto c = [&](int tn, int tm) {
    const int64_t tiles = a.offsets ? a.M / tm + (E < a.M ? E : a.M) : (a.M + tm - 1) / tm;
    return tiles * ((a.N + tn - 1) / tn);
  };
  if (a.M <= 16 * E || c(32, 16) <= 256) {
    if (c(16, 16) <= 128 && a.K >= 2048) return launch_stream<1, 1, 8, 4, BYTES>(a, s);
    if (c(64, 16) < 1024) return launch_stream<2, 1, 2, 4, BYTES>(a, s);
    return launch_stream<4, 1, 2, 2, BYTES>(a, s);
  }
  if (a.M <= 32 * E || c(64, 32) <= 256) {
    if (c(32, 32) <= 256) return launch_stream<2, 2, 2, 4, BYTES>(a, s);
    return launch_stream<4, 2, 2, 2, BYTES>(a, s);
  }
  if (a.M <= 64 * E || c(64, 64) <= 512) {
    if (c(64, 64) < 1024) return launch_stream<4, 4, 4, 2, BYTES>(a, s);
    return launch_stream<4, 4, 2, 2, BYTES>(a, s);
  }
  if (a.M >= 192 * E && size > 128 * unit) return launch_cfg<4, 4, 4, 4, BYTES, 2>(a, s);
  if (a.M >= 64 * E && size >= 24 * unit) {
    if (c(128, 128) <= 256) return launch_cfg<2, 4, 4, 2, BYTES, 4>(a, s);
    return launch_cfg<2, 4, 4, 2, BYTES, 2>(a, s);
  }
  return launch_cfg<2, 2, 4, 2, BYTES, 2>(a, s);
}

}  // namespace

hipError_t launch_linear_scaled(const ScaledArgs& a, hipStream_t s) {
  return a.bits == 8 ? launch_bytes<1>(a, s) : launch_bytes<2>(a, s);
}

}  // namespace ilw
