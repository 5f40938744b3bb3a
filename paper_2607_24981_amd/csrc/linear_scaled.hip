// linear_scaled.hip -- int8 products with a scale for each token and a factor for
// each channel, dense or grouped by expert, int16 or int8 out.
//
//   y[m][n] = sat(floor((floor(acc F / 2^max(q - 4, 0)) + b + 8) / 16))
// F = floor(X Y / 2^32) of the token's scale X = S 2^z in [2^31, 2^32) and the
// channel's multiplier Y = mult 2^u in [2^30, 2^31), so that F is in [2^29, 2^31)
// and keeps 29 bits or more whatever the scales are; q = shift + z + u - 18.  From
// q = 36 on floor(acc F / 2^(q - 4)) is the product's high word shifted right: two
// 32-bit high products, two adds, two shifts and a median a value.  Below, the
// 64-bit product is shifted (q of a layer whose outputs use their bits is 37 and
// more: acc of 13 bits, F of 30, outputs of 6).
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
// One output before saturation; FAST: q >= 36.
template <bool FAST>
__device__ __forceinline__ int32_t scaled(int32_t acc, const Channel& c, const Token& t) {
  const int32_t F = (int32_t)__umulhi(t.X, c.Y);
  const int32_t s = c.q + t.z;
  if (FAST) return ((__mulhi(acc, F) >> min(s - 32, 31)) + c.c) >> 4;
  const int64_t v = (((int64_t)acc * F) >> min(max(s, 0), 63)) + c.c;
  return (int32_t)min(max(v >> 4, (int64_t)-65536), (int64_t)65536);
}

template <int WN, int WM, int FI, int FJ, int BYTES, bool KTAIL>
__global__ __launch_bounds__(64 * WN * WM) void scaled_kernel(ScaledArgs a, uint32_t tiles_n) {
  using Product = TileProduct<WN, WM, FI, FJ, KTAIL>;
  constexpr int WTN = Product::WTN, WTM = Product::WTM, TN = Product::TN, TM = Product::TM,
                NT = Product::NT, STAGE = Product::STAGE;
  constexpr int OSTR = TN * BYTES / 4 + 4;  // words per staged token row
  constexpr int SOUT = TM * OSTR * 4;
  __shared__ __attribute__((aligned(1024))) int8_t sbuf[2 * STAGE > SOUT ? 2 * STAGE : SOUT];
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
          v[r] = min(max(scaled<decltype(fast)::value>(p.acc[i][j][r], ch[r], tok), -lim), lim);
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
  if (least_q + least_z >= 32) scale(Flag<true>{});
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

template <int WN, int WM, int FI, int FJ, int BYTES>
hipError_t launch_cfg(const ScaledArgs& a, hipStream_t s) {
  constexpr int TN = 16 * FI * WN, TM = 16 * FJ * WM;
  const uint32_t tiles_n = (uint32_t)((a.N + TN - 1) / TN);
  const int64_t tiles_m =
      a.offsets ? a.M / TM + (a.E < a.M ? a.E : a.M) : (a.M + TM - 1) / TM;
  // below 2^32 threads: the entry point holds (M / 64 + E) (N / 128 + 1) below 2^22,
  // and the one tile of 1024 threads has E <= M / 192
  const dim3 grid((unsigned)(tiles_m * tiles_n)), block(64 * WN * WM);
  if (a.K % KB == 0)
    hipLaunchKernelGGL((scaled_kernel<WN, WM, FI, FJ, BYTES, false>), grid, block, 0, s, a, tiles_n);
  else
    hipLaunchKernelGGL((scaled_kernel<WN, WM, FI, FJ, BYTES, true>), grid, block, 0, s, a, tiles_n);
  return hipGetLastError();
}

template <int BYTES>
hipError_t launch_bytes(const ScaledArgs& a, hipStream_t s) {
  const int64_t size = a.M * a.N, unit = 65536;
  if (a.M >= 192 * (int64_t)a.E && size > 128 * unit) return launch_cfg<4, 4, 4, 4, BYTES>(a, s);
  if (a.M >= 64 * (int64_t)a.E && size >= 24 * unit) return launch_cfg<2, 4, 4, 2, BYTES>(a, s);
  if (a.M <= 16 * (int64_t)a.E && a.E * (int64_t)((a.N + 255) / 256) >= 512)
    return launch_cfg<4, 1, 4, 2, BYTES>(a, s);
  return launch_cfg<2, 2, 4, 2, BYTES>(a, s);
}

}  // namespace

hipError_t launch_linear_scaled(const ScaledArgs& a, hipStream_t s) {
  return a.bits == 8 ? launch_bytes<1>(a, s) : launch_bytes<2>(a, s);
}

}  // namespace ilw
