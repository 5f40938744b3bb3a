// grouped.hip -- int8 linear layers grouped by expert: rows sorted by expert,
// each expert its own weights, ragged numbers of rows.
//
//   y[m][n] = sat8(rq(b[e][n] + sum_k x[r(m)][k] w[e][n][k]; rq[e][n]))
//
// Tiles and their sums: expert_tiles.h.
#include "decoder_internal.h"
#include "expert_tiles.h"

namespace ilw {
namespace {

template <int WN, int WM, int FI, int FJ, bool KTAIL>
__global__ __launch_bounds__(64 * WN * WM) void grouped_kernel(GroupedArgs a, uint32_t tiles_n) {
  using Product = TileProduct<WN, WM, FI, FJ, KTAIL>;
  constexpr int WTN = Product::WTN, WTM = Product::WTM, TN = Product::TN, TM = Product::TM,
                NT = Product::NT, STAGE = Product::STAGE;
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
  Product p;
  p.start(a, tl, sbuf, tid);
  bool clamp_acc = false;
  for (int c = tid; c < TN; c += NT) {
    const int64_t n = (int64_t)tl.e * N + min(n0 + c, N - 1), q = a.nq == 1 ? 0 : n;
    RqI64 r;
    clamp_acc |= !r.init_bounded(a.mult[q], a.shift[q], a.bias ? a.bias[n] : 0, (uint32_t)K << 14);
    rqc[c] = r;
  }
  if (tid == 0) unbounded = 0;
  p.ready();
  if (clamp_acc) unbounded = 1;  // (published by the loop's barriers)
  p.run();

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
          const int32_t v = dead[j] ? 0 : p.acc[i][j][r];
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
