// quantize_rows.hip -- int16 rows to int8 codes with a scale for each row.
//
// With A the largest magnitude of a row, S = max(1, ceil(2^14 A / 127)) and
// X = 2^14 x, a code is floor((2 X + S) / (2 S)) = floor(X / S + 1/2), in [-127, 127].
// Values and scale are shifted left by e so that A 2^e is in [2^14, 2^15] (S 2^e
// then in [2^21.01, 2^22.02]), and with R = 2^53 / (S 2^e) to the nearest, below
// 2^32, the code is bits 40 .. 47 of
//   2 (x 2^e) R + 2^39 + 2^15 + 1:
// the rounding of R moves X / S by at most 2^15 1/2 2 / 2^40 (and 2^-17 of that for
// the reciprocal's own error), so the sum is above the true value by less than
// 2^17 / 2^40 = 2^-23, and (2 X + S) / (2 S), a multiple of 1 / (2 S) >= 2^-23.02
// (S 2^e counted), meets no integer on the way.  x enters as x + 2^15, an unsigned
// 16-bit half of a word, with the offset's product taken off the addend modulo 2^64.
//
// Bound: bytes (16000 rows of 4096 values: 35 us; 197 MB take 39 to copy).  TPR lanes
// take a row, 16 values a unit, up to three units a lane (the widest: four) in
// registers, so that a row is read once up to 16384 values.
#include "step_internal.h"

namespace ilw {
namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Unit {  // 16 values
  u32x4 a, b;
};
__device__ __forceinline__ Unit load_unit(const int16_t* p) {
  return {*(const u32x4*)p, *(const u32x4*)(p + 8)};
}

// Largest and lowest value of pairs, both halves apart.
struct Range {
  s16x2 hi, lo;
  __device__ __forceinline__ void add(const Unit& u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = u.a[i], b = u.b[i];  // (bit_cast of an element itself takes the first)
      const s16x2 p = __builtin_bit_cast(s16x2, a), q = __builtin_bit_cast(s16x2, b);
      hi = __builtin_elementwise_max(hi, __builtin_elementwise_max(p, q));
      lo = __builtin_elementwise_min(lo, __builtin_elementwise_min(p, q));
    }
  }
  __device__ __forceinline__ int32_t magnitude() const {
    return max(max((int32_t)hi.x, (int32_t)hi.y), -min((int32_t)lo.x, (int32_t)lo.y));
  }
};

// The codes of a row whose largest magnitude is A.
struct Codes {
  uint32_t R;
  int32_t e1;  // e + 1
  uint64_t c;
  __device__ __forceinline__ int32_t init(int32_t A) {  // the row's scale
    const int32_t S = A ? (int32_t)((((uint32_t)A << 14) + 126u) / 127u) : 1;
    if (A == 0) A = 1;  // (every x is 0: any scale gives 0)
    const int32_t e = max(__clz(A) - 17, 0);
    const double d = (double)((A == 1 ? 130 : S) << e);  // 130: the scale of A = 1
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
    r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
    R = (uint32_t)__builtin_fma(0x1p53, r, 0.5);
    e1 = e + 1;
    c = ((uint64_t)1 << 39) + (1 << 15) + 1 - ((uint64_t)R << (15 + e1));
    return S;
  }
  // the high word whose byte 1 is the code of h - 2^15, h in [0, 2^16)
  __device__ __forceinline__ uint32_t word(uint32_t h) const {
    return (uint32_t)(((uint64_t)(h << e1) * R + c) >> 32);
  }
  __device__ __forceinline__ uint32_t pack(uint32_t p, uint32_t q) const {  // four values
    p ^= 0x80008000u;
    q ^= 0x80008000u;
    const uint32_t lo = __builtin_amdgcn_perm(word(p >> 16), word(p & 0xffff), 0x0c0c0501u);
    const uint32_t hi = __builtin_amdgcn_perm(word(q >> 16), word(q & 0xffff), 0x0c0c0501u);
    return lo | (hi << 16);
  }
  __device__ __forceinline__ u32x4 unit(const Unit& u) const {
    return u32x4{pack(u.a[0], u.a[1]), pack(u.a[2], u.a[3]), pack(u.b[0], u.b[1]),
                 pack(u.b[2], u.b[3])};
  }
};

constexpr int NT = 256;

template <int TPR>
__global__ __launch_bounds__(NT) void quantize_kernel(QuantizeArgs a) {
  constexpr int RPB = NT / TPR;  // rows a workgroup
  constexpr int UNITS = TPR == NT ? 4 : 3;  // a lane keeps
  const int tid = threadIdx.x, t = tid % TPR;
  const int64_t m = (int64_t)blockIdx.x * RPB + tid / TPR;
  if (TPR < NT && m >= a.M) return;  // (no barrier below for these)
  const int32_t units = a.K / 16;
  const int16_t* x = a.x + m * a.ld;
  int8_t* y = a.y + m * a.K;
  Unit u[UNITS];
  Range r = {{0, 0}, {0, 0}};
#pragma unroll
  for (int i = 0; i < UNITS; ++i)
    if (t + i * TPR < units) u[i] = load_unit(x + (t + i * TPR) * 16);
#pragma unroll
  for (int i = 0; i < UNITS; ++i)
    if (t + i * TPR < units) r.add(u[i]);
  if (TPR == NT)
    for (int32_t i = t + UNITS * TPR; i < units; i += TPR) r.add(load_unit(x + (int64_t)i * 16));
  int32_t A = r.magnitude();
#pragma unroll
  for (int o = 1; o < (TPR < 64 ? TPR : 64); o <<= 1) A = max(A, __shfl_xor(A, o, 64));
  if (TPR > 64) {
    __shared__ int32_t part[NT / 64];
    if ((tid & 63) == 0) part[tid >> 6] = A;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) A = max(A, part[i]);
  }
  Codes q;
  const int32_t S = q.init(A);
  if (t == 0) a.scale[m] = S;
#pragma unroll
  for (int i = 0; i < UNITS; ++i)
    if (t + i * TPR < units) *(u32x4*)(y + (t + i * TPR) * 16) = q.unit(u[i]);
  if (TPR == NT)
    for (int32_t i = t + UNITS * TPR; i < units; i += TPR)
      *(u32x4*)(y + (int64_t)i * 16) = q.unit(load_unit(x + (int64_t)i * 16));
}

template <int TPR>
hipError_t launch(const QuantizeArgs& a, hipStream_t s) {
  constexpr int RPB = NT / TPR;
  const int64_t blocks = (a.M + RPB - 1) / RPB;
  hipLaunchKernelGGL((quantize_kernel<TPR>), dim3((unsigned)blocks), dim3(NT), 0, s, a);
  return hipGetLastError();
}

// Lanes a row: as many as have two units each, or three where there is much to read.
// In us, 4, 3 or 2 units a lane: 8000 rows of 256 values 3.9, 3.1 with 2; 40000 rows of
// 640 16.5 with 3, 18.2 with 2, 8000 rows 5.4 and 5.5; 1000 rows of 1024 3.5 with 4, 2.5
// with 1; 16000 rows of 4096 34.3 with 4, 31.6 with 1.  1 unit a lane leaves lanes idle
// (40000 rows of 512: 17.2, 13.3 with 2).
int lanes_of(const QuantizeArgs& a) {
  const int32_t units = a.K / 16, most = a.M >= ((int64_t)1 << 24) / a.K ? 3 : 2;
  if (units <= 4 * most) return 4;
  if (units <= 16 * most) return 16;
  return units <= 64 * most ? 64 : NT;
}

}  // namespace

bool quantize_rows_fits(const QuantizeArgs& a) {
  return a.M < ((int64_t)1 << 32) / lanes_of(a) - NT;
}

hipError_t launch_quantize_rows(const QuantizeArgs& a, hipStream_t s) {
  switch (lanes_of(a)) {
    case 4: return launch<4>(a, s);
    case 16: return launch<16>(a, s);
    case 64: return launch<64>(a, s);
    default: return launch<NT>(a, s);
  }
}

}  // namespace ilw
