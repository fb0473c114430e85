// Kernels of the decoder loop's dense path in 8 bits: blocks of e4m3 codes made
// from rows, the residual's addition and root-mean-square norm with an output in
// such blocks, and the product of two matrices that are kept in them.  Stateless
// entry points: every buffer is the caller's, every call is enqueued on the
// caller's stream.
//
// A value is an e4m3 code times a power of two that 128 columns of a row, or of
// 128 rows, share.  Codes are floating numbers themselves, so a scale that is no
// power of two would add range and no precision, and a power of two multiplies
// exactly wherever it is applied: here in the conversion of codes to bf16
// (v_cvt_scalef32_pk_bf16_fp8), which holds every code times a power of two.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <iterator>

#include "device.h"
#include "kernels.h"
#include "moesplit.h"

namespace {

using msk::overlap;

constexpr int kBlock = 128;  // columns that share a scale, and rows of a weight's block
constexpr int kExpBias = 127;
constexpr int kExpMin = -40, kExpMax = 40;
constexpr float kCodeMax = 448.0f;
constexpr int kMostColumns = 16384;
constexpr int kMostOutputs = 1 << 25, kMostRows = 1 << 24;  // of a launch

__device__ __forceinline__ uint32_t bf16_bits(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));  // to nearest even, NaN stays NaN
}

// 2^e, e in [-126, 127]
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ float load_value(float x) { return x; }
__device__ __forceinline__ float load_value(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

// Eight consecutive values, 16-byte aligned.
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// the value to convert: within the codes' range, NaN for what is not finite
__device__ __forceinline__ float code_range(float x) {
  return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? fminf(fmaxf(x, -kCodeMax), kCodeMax) : __uint_as_float(0x7fc00000u);
}

__device__ __forceinline__ uint2 codes8(const float (&v)[8]) {
  int c[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    c[i] = __builtin_amdgcn_cvt_pk_fp8_f32(code_range(v[4 * i]), code_range(v[4 * i + 1]), 0, false);
    c[i] = __builtin_amdgcn_cvt_pk_fp8_f32(code_range(v[4 * i + 2]), code_range(v[4 * i + 3]), c[i], true);
  }
  return make_uint2(static_cast<uint32_t>(c[0]), static_cast<uint32_t>(c[1]));
}

// The exponent of a block from the bits of its largest finite magnitude m 2^x, 1 <= m < 2:
// 448 = 1.75 * 2^8; zero and subnormal magnitudes end at kExpMin.
__device__ __forceinline__ int block_exponent(uint32_t top) {
  return min(max(static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u), kExpMin), kExpMax);
}

__device__ __forceinline__ uint32_t finite_magnitude(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0;
}

__device__ __forceinline__ uint32_t max_of_lanes(uint32_t v, int lanes) {  // groups of `lanes`
  for (int s = lanes / 2; s >= 1; s >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), s, 64)));
  return v;
}

// ----------------------------------------------------------------- rows to blocks
//
// Sixteen lanes take 128 columns of a row, eight values each.  Blocks of one row are theirs; one
// of 128 rows is a work-group's, its values in registers until its largest magnitude is known.
// Bound by the bytes: 32000 x 4096 from bf16 (393 MB) 80 us, 4.9 TB/s, as fast as a copy; 4096
// x 4096 10.9; a row of 4096 2.1.
constexpr int kQuantThreads = 256;

template <typename X>
__global__ __launch_bounds__(kQuantThreads) void quant_rows_kernel(const X* __restrict__ x, int rows, int n, int nb,
                                                                   uint8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  const int64_t b = (static_cast<int64_t>(blockIdx.x) * kQuantThreads + threadIdx.x) / 16;  // block: row b / nb
  const int row = static_cast<int>(b / nb), kb = static_cast<int>(b % nb), k = kb * kBlock + 8 * (threadIdx.x & 15);
  const bool in = row < rows && k < n;
  const size_t at = static_cast<size_t>(row) * n + k;
  float v[8] = {};
  if (in) load8(x + at, v);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[i]));
  const int e = block_exponent(max_of_lanes(top, 16));
  if (!in) return;
  const float scale = pow2(-e);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= scale;
  *reinterpret_cast<uint2*>(codes + at) = codes8(v);
  if ((threadIdx.x & 15) == 0) exps[b] = static_cast<uint8_t>(e + kExpBias);
}

template <typename X>
__global__ __launch_bounds__(kQuantThreads) void quant_blocks_kernel(const X* __restrict__ x, int rows, int n, int nb,
                                                                     uint8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  constexpr int PER = kBlock * 16 / kQuantThreads;  // pieces of eight values per thread
  __shared__ uint32_t tops[kQuantThreads / 64];
  const int r0 = static_cast<int>(blockIdx.x / nb) * kBlock + threadIdx.x / 16;
  const int k = static_cast<int>(blockIdx.x % nb) * kBlock + 8 * (threadIdx.x & 15);
  float v[PER][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = r0 + i * (kQuantThreads / 16);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    if (r < rows && k < n) load8(x + static_cast<size_t>(r) * n + k, v[i]);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, finite_magnitude(v[i][j]));
  top = max_of_lanes(top, 64);
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / 64; ++w) top = max(top, tops[w]);
  const int e = block_exponent(top);
  const float scale = pow2(-e);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = r0 + i * (kQuantThreads / 16);
    if (r >= rows || k >= n) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= scale;
    *reinterpret_cast<uint2*>(codes + static_cast<size_t>(r) * n + k) = codes8(v[i]);
  }
  if (threadIdx.x == 0) exps[blockIdx.x] = static_cast<uint8_t>(e + kExpBias);
}

// ------------------------------------------------------------ residual and norm
//
// One to four waves per row, sixteen lanes to 128 columns; the sum h + y stays in registers
// between its two uses.  The sum of squares and the norm are in double precision, and each value
// is rounded once, to an fp32 that leaves the second rounding to bf16 or a code exact: a code is
// the nearest to the exact normalised value, and no exponent depends on how fp32 would have
// rounded next to a power of two.  2048 x 4096 with a bf16 y, gain, running sum and codes (75 MB)
// 21 us, 3.6 TB/s, and 4096 rows 33; with an fp32 y and no running sum 17.  Between the bytes (15
// us) and the double precision's instructions: the exponents chosen and codes made in it too
// took 27.  A row of 4096 3.7 us: latency.
constexpr int kNormThreads = 256;

// d as fp32 that a second rounding, to bf16 or a code, cannot tell from d, nor a comparison
// with a number of fewer bits: of the two neighbours the one with an odd last bit where d is
// neither.  (Finite numbers stay finite.)
__device__ __forceinline__ float to_odd(double d) {
  const float f = static_cast<float>(d);
  const double e = d - f;
  const int u = static_cast<int>(__float_as_uint(f));
  const int away = ((__double2hiint(e) ^ u) >> 31) | 1;  // towards d
  return (e < 0.0 || e > 0.0) && !(u & 1) ? __uint_as_float(static_cast<uint32_t>(u + away)) : f;
}

__device__ __forceinline__ uint4 pack_bf16(const float (&f)[8]) {
  return make_uint4(bf16_bits(f[0]) | bf16_bits(f[1]) << 16, bf16_bits(f[2]) | bf16_bits(f[3]) << 16,
                    bf16_bits(f[4]) | bf16_bits(f[5]) << 16, bf16_bits(f[6]) | bf16_bits(f[7]) << 16);
}

struct NormArgs {
  const uint16_t* h;
  const void* y;
  const uint16_t* weight;
  uint16_t *sum_out, *out;
  uint8_t *codes, *exps;
  double eps;
  int T, d, nb;
};

template <typename Y, int WAVES, int PER>
__global__ __launch_bounds__(kNormThreads) void residual_norm_q_kernel(NormArgs a) {
  constexpr int LANES = 64 * WAVES;
  __shared__ double sums[kNormThreads / 64];
  const int lane = threadIdx.x % LANES, t = blockIdx.x * (kNormThreads / LANES) + threadIdx.x / LANES;
  const int d = t < a.T ? a.d : 0;  // columns of the row
  const size_t row = static_cast<size_t>(t) * a.d;
  const Y* y = static_cast<const Y*>(a.y);
  double x[PER][8], ss = 0.0;
#pragma unroll
  for (int m = 0; m < PER; ++m) {
    const int k = 8 * (lane + m * LANES);
    float h[8] = {}, r[8] = {};
    if (k < d) {
      load8(a.h + row + k, h);
      if (y) load8(y + row + k, r);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[m][i] = static_cast<double>(h[i]) + r[i];
  }
#pragma unroll
  for (int m = 0; m < PER; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fma(x[m][i], x[m][i], ss);
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) ss += __shfl_xor(ss, s, 64);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = ss;
    __syncthreads();
    ss = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) ss += sums[threadIdx.x / LANES * WAVES + w];
  }
  const double inv = 1.0 / sqrt(ss / a.d + a.eps);
#pragma unroll
  for (int m = 0; m < PER; ++m) {
    const int piece = lane + m * LANES, k = 8 * piece;
    const bool in = k < d;
    float f[8];
    if (in && a.sum_out) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_odd(x[m][i]);
      *reinterpret_cast<uint4*>(a.sum_out + row + k) = pack_bf16(f);
    }
    if (a.weight) {
      float g[8] = {};
      if (in) load8(a.weight + k, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_odd(x[m][i] * (inv * g[i]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_odd(x[m][i] * inv);
    }
    if (in && a.out) *reinterpret_cast<uint4*>(a.out + row + k) = pack_bf16(f);
    if (!a.codes) continue;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, in ? finite_magnitude(f[i]) : 0u);
    const int e = block_exponent(max_of_lanes(top, 16));
    if (!in) continue;
    const float scale = pow2(-e);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= scale;
    *reinterpret_cast<uint2*>(a.codes + row + k) = codes8(f);
    if ((threadIdx.x & 15) == 0) a.exps[static_cast<size_t>(t) * a.nb + piece / 16] = static_cast<uint8_t>(e + kExpBias);
  }
}

// ----------------------------------------------------------------------- product

struct DenseArgs {
  const uint8_t *x, *x_exp, *w, *w_exp;
  const void* add;
  void* y;
  int T, n_in, n_out, nb;
};

// Sixteen codes -> two operands of eight bf16, times 2^e.
__device__ __forceinline__ void to_bf16(uint4 c, float scale, msk::bf16x8_t (&o)[2]) {
  auto pair = [&](uint32_t u, bool high) {
    return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(u), scale, true)
                                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(u), scale, false));
  };
  o[0] = msk::as_bf16x8(make_uint4(pair(c.x, false), pair(c.x, true), pair(c.y, false), pair(c.y, true)));
  o[1] = msk::as_bf16x8(make_uint4(pair(c.z, false), pair(c.z, true), pair(c.w, false), pair(c.w, true)));
}

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(uint16_t* p, float v) { *p = static_cast<uint16_t>(bf16_bits(v)); }

constexpr uint32_t scale_bits(int e) { return static_cast<uint32_t>(e + kExpBias); }

// a stored exponent, kept in range whatever the byte holds
__device__ __forceinline__ uint32_t exponent_in_range(uint32_t x) {
  return min(max(x, scale_bits(kExpMin)), scale_bits(kExpMax));
}
__device__ __forceinline__ float scale_of(uint32_t x) { return __uint_as_float(x << 23); }

__device__ const uint4 kZeroCodes = {0, 0, 0, 0};

// Four neighbouring outputs of a token.
template <typename Y>
__device__ __forceinline__ void store4(const DenseArgs& a, int t, int o, msk::f32x4_t v, int vec) {
  const size_t i = static_cast<size_t>(t) * a.n_out + o;
  Y* y = static_cast<Y*>(a.y) + i;
  const Y* add = a.add ? static_cast<const Y*>(a.add) + i : nullptr;
  if (!vec) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (o + r < a.n_out) store_value(y + r, v[r] + (add ? load_value(add[r]) : 0.0f));
  } else if (o < a.n_out) {  // n_out a multiple of 4, rows aligned to four values
    if constexpr (sizeof(Y) == 4) {
      float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
      if (add) b = *reinterpret_cast<const float4*>(add);
      *reinterpret_cast<float4*>(y) = make_float4(v[0] + b.x, v[1] + b.y, v[2] + b.z, v[3] + b.w);
    } else {
      uint2 b = make_uint2(0, 0);
      if (add) b = *reinterpret_cast<const uint2*>(add);
      v[0] += __uint_as_float(b.x << 16), v[1] += __uint_as_float(b.x & 0xffff0000u);
      v[2] += __uint_as_float(b.y << 16), v[3] += __uint_as_float(b.y & 0xffff0000u);
      *reinterpret_cast<uint2*>(y) = make_uint2(bf16_bits(v[0]) | bf16_bits(v[1]) << 16, bf16_bits(v[2]) | bf16_bits(v[3]) << 16);
    }
  }
}

// Eight.
template <typename Y>
__device__ __forceinline__ void store8(const DenseArgs& a, int t, int o, msk::f32x4_t u, msk::f32x4_t v, int vec) {
  const size_t i = static_cast<size_t>(t) * a.n_out + o;
  if (sizeof(Y) == 4 || !vec || a.n_out % 8 != 0 || ((reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.add)) & 15)) {
    store4<Y>(a, t, o, u, vec);
    store4<Y>(a, t, o + 4, v, vec);
  } else if (o < a.n_out) {
    float f[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]}, b[8] = {};
    if (a.add) load8(static_cast<const uint16_t*>(a.add) + i, b);
#pragma unroll
    for (int r = 0; r < 8; ++r) f[r] += b[r];
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + i) = pack_bf16(f);
  }
}

// Few tokens: MO blocks of 16 outputs x NT of 16 tokens (the last one repeated) per
// work-group, its KW waves every KW-th 128 columns.  Codes go from memory to registers: lane l has
// pieces l / 16 and 4 + l / 16 of sixteen codes of row l % 16.
//   Bound by latency: a turn's loads are all waited for before they are converted, so a wave makes as
// many trips to memory as it has turns (4096 columns, eight waves: four).  One token 4096 -> 6144 7.5
// us, 3.4 TB/s; 4096 -> 32000 24.5, 5.3 TB/s; 61 tokens 2000 -> 5003 8.4-9.1.
template <typename Y, int KW, int MO, int NT>
__global__ __launch_bounds__(64 * KW) void dense_q_few_kernel(DenseArgs a, int vec) {
  __shared__ __align__(16) float red[KW][MO * NT][64][4];
  const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int o0 = blockIdx.x * 16 * MO;  // (MO a power of two: of one block of 128)
  const uint8_t* w_exp = a.w_exp + static_cast<size_t>(o0 / kBlock) * a.nb;
  const uint8_t *w[MO], *x[NT], *x_exp[NT];
#pragma unroll
  for (int m = 0; m < MO; ++m) w[m] = a.w + static_cast<size_t>(min(o0 + 16 * m + r16, a.n_out - 1)) * a.n_in;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const size_t t = min(16 * n + r16, a.T - 1);
    x[n] = a.x + t * a.n_in, x_exp[n] = a.x_exp + t * a.nb;
  }
  msk::f32x4_t acc[MO][NT];
#pragma unroll
  for (int m = 0; m < MO; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = msk::f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int b = wv; b < a.nb; b += KW) {
    uint4 cw[MO][2], cx[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = b * kBlock + 16 * (4 * h + g4);
      const bool in = k < a.n_in;
#pragma unroll
      for (int m = 0; m < MO; ++m) cw[m][h] = in ? *reinterpret_cast<const uint4*>(w[m] + k) : kZeroCodes;
#pragma unroll
      for (int n = 0; n < NT; ++n) cx[n][h] = in ? *reinterpret_cast<const uint4*>(x[n] + k) : kZeroCodes;
    }
    const float sw = scale_of(exponent_in_range(w_exp[b]));
    float sx[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) sx[n] = scale_of(exponent_in_range(x_exp[n][b]));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      msk::bf16x8_t A[MO][2], B[2];
#pragma unroll
      for (int m = 0; m < MO; ++m) to_bf16(cw[m][h], sw, A[m]);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        to_bf16(cx[n][h], sx[n], B);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int m = 0; m < MO; ++m) acc[m][n] = msk::mfma16(A[m][q], B[q], acc[m][n]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MO; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) *reinterpret_cast<msk::f32x4_t*>(red[wv][m * NT + n][lane]) = acc[m][n];
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * MO * NT; i += 64 * KW) {
    const int p = i / 64, l = i & 63, t = 16 * (p % NT) + (l & 15);
    msk::f32x4_t v = *reinterpret_cast<const msk::f32x4_t*>(red[0][p][l]);
#pragma unroll
    for (int k = 1; k < KW; ++k) v += *reinterpret_cast<const msk::f32x4_t*>(red[k][p][l]);
    if (t < a.T) store4<Y>(a, t, o0 + 16 * (p / NT) + 4 * (l >> 4), v, vec);
  }
}

// Some tokens: y^T = W x^T, a work-group takes BM tokens x BN outputs; both operands go to LDS as
// codes by direct loads (a row's 128 columns of a stage are a cache line; piece p of sixteen
// codes of row r sits in slot p ^ (r % 8), so the lanes that an LDS read serves together hit
// distinct banks), in a ring of NST stages.  WM x WN waves split the tile, and KS times as many
// the stages, each part with a ring of its own; the parts' sums are added in LDS in the end.
//   An fp32 result: codes become bf16, times their scale, as operands are read; every
// product is exact and sums are fp32.  A bf16 result (EIGHT): the matrix cores take the codes
// and the scales as they are, at twice the rate.  Of the products of eight neighbouring columns they
// cut all to multiples of 2^-13 of the power of two that the largest sum of two codes' exponents
// gives (subnormal codes count as 2^-6, zero products not), then add them, and the groups' sums in fp32.
// Only products whose exponents are 8 and more below lose anything: 1.5e-5 of a result of normal
// values, a hundredth of what its rounding to bf16 takes and too much for an fp32 one; less than 2^-10
// of the largest where no code is subnormal, a quarter of what that rounding takes at most.
//   Bound by the latency of a stage (loads, a barrier, LDS reads, then few matrix instructions
// of a wave), so one that has the CU to itself takes its stages several at a time: with 1, 2 and 4
// parts a round of tiles of 32 x 32 at 4096 columns takes 12.4, 9.6 and 8.8 us with fp32 results and
// 8.8, 7.3 and 6.8 with bf16 ones, of 64 x 64 18.9, 15.5 and 14.1, and 12.3, 10.7 and 10.6; two
// rounds of 32 x 32 14.2, 12.6 and 15.8 (the same inputs again and again).  64 tokens 4096 -> 4096 8.9
// and 7.3 us, 512 tokens 4096 -> 6144 35 and 22.6 (three sets of inputs in turn).
constexpr int kStageLoad = 64 * 16;      // one load: 8 rows
constexpr int kRows16 = 16 * kBlock;     // bytes of 16 staged rows
constexpr int kTileExps = 16384;         // exponents of a tile's tokens that fit: blocks of columns x BM

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// Tile w of a launch: an XCD takes neighbouring ones, and of up to four blocks of tokens the
// blocks of outputs follow each other, so that the tiles of a moment share both.
__device__ __forceinline__ int2 tile_of(int w, int n, int m_tiles) {
  const int i = msk::xcd_local(w, n), wide = n / m_tiles, band = 4 * wide;
  const int m0 = i / band * 4, rows = min(m_tiles - m0, 4), at = i % band;
  return make_int2(m0 + at % rows, at / rows);
}

// The exponents of a tile's tokens t0 .. t0 + BM - 1, put(token, block of columns, exponent): the
// rows follow each other in memory, and eight are requested before the first is used.
template <int BM, int THREADS, typename Put>
__device__ __forceinline__ void stage_exponents(const DenseArgs& a, int t0, Put put) {
  const uint8_t* e = a.x_exp + static_cast<size_t>(t0) * a.nb;
  const int n = min(BM, a.T - t0) * a.nb;
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * THREADS) {
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e[min(i0 + i * THREADS, n - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i0 + i * THREADS < n)
        put((i0 + i * THREADS) / a.nb, (i0 + i * THREADS) % a.nb, static_cast<uint8_t>(exponent_in_range(v[i])));
  }
}

template <typename Y, bool EIGHT, int BM, int BN, int WM, int WN, int NST, int KS>
__global__ __launch_bounds__(64 * WM * WN * KS) void dense_q_tile_kernel(DenseArgs a, int m_tiles, int vec) {
  constexpr int NWV = WM * WN;
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // 16-wide blocks per wave
  constexpr int NL = (BM + BN) / 8 / NWV;              // loads per wave and stage
  constexpr int SBYTES = (BM + BN) * kBlock;
  constexpr int WB = (BN + kBlock - 1) / kBlock + 1;   // weights' scales that a tile may touch
  constexpr int EXPS = BM * (kMostColumns / kBlock) < kTileExps ? BM * (kMostColumns / kBlock) : kTileExps;
  static_assert(TM * WM * 16 == BM && TN * WN * 16 == BN && NL * 8 * NWV == BM + BN, "tile split");
  static_assert(NST >= 2 && KS * NST * SBYTES + EXPS + WB * (kMostColumns / kBlock) <= 160 * 1024 && (NST - 2) * NL < 64, "ring");
  __shared__ __align__(16) unsigned char lds[KS * NST * SBYTES];
  __shared__ uint8_t xe[EXPS], we[WB * (kMostColumns / kBlock)];  // [blocks of columns][BM], [WB][blocks of columns]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wv = wave % NWV, part = wave / NWV;  // of the waves that take stages part, part + KS, ...
  const int wm = wv % WM, wn = wv / WM;
  const int2 tile = tile_of(blockIdx.x, gridDim.x, m_tiles);
  const int t0 = tile.x * BM, o0 = tile.y * BN;
  const int lrow = lane >> 3, lk = 16 * ((lane & 7) ^ lrow);
  const uint8_t* src[NL];  // staged rows: the tile's BM tokens, then its BN outputs
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int r = 8 * (wv + NWV * j) + lrow;
    src[j] = (r < BM ? a.x + static_cast<size_t>(min(t0 + r, a.T - 1)) * a.n_in
                     : a.w + static_cast<size_t>(min(o0 + r - BM, a.n_out - 1)) * a.n_in) + lk;
  }
  unsigned char* const ring = lds + part * NST * SBYTES;
  const uint32_t lbase = msk::lds_address(lds) + part * NST * SBYTES + wv * kStageLoad;
  auto issue = [&](int turn, int buf) {  // stages past the last reload it (in bounds, never read)
    const int k0 = min(turn * KS + part, a.nb - 1) * kBlock;
    if (k0 + kBlock <= a.n_in) {
#pragma unroll
      for (int j = 0; j < NL; ++j) msk::lds_load16(src[j] + k0, lbase + buf * SBYTES + NWV * j * kStageLoad);
    } else {  // zeros past the rows' ends: what follows in memory may be NaN
#pragma unroll
      for (int j = 0; j < NL; ++j)
        msk::lds_load16(k0 + lk < a.n_in ? src[j] + k0 : reinterpret_cast<const uint8_t*>(&kZeroCodes),
                        lbase + buf * SBYTES + NWV * j * kStageLoad);
    }
  };
#pragma unroll
  for (int p = 0; p < NST - 1; ++p) issue(p, p);
  stage_exponents<BM, 64 * NWV * KS>(a, t0, [&](int r, int b, uint8_t e) { xe[b * BM + r] = e; });
  const int wb0 = o0 / kBlock, wbn = (a.n_out - 1) / kBlock;
  for (int i = threadIdx.x; i < WB * a.nb; i += 64 * NWV * KS)
    we[i] = static_cast<uint8_t>(exponent_in_range(a.w_exp[static_cast<size_t>(min(wb0 + i / a.nb, wbn)) * a.nb + i % a.nb]));
  int fo[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) fo[h] = (lane & 15) * kBlock + 16 * ((4 * h + (lane >> 4)) ^ (lane & 7));
  int wb[TN];  // the scale's row of each block of outputs
#pragma unroll
  for (int n = 0; n < TN; ++n) wb[n] = ((o0 + (wn * TN + n) * 16) / kBlock - wb0) * a.nb;
  const uint8_t* xel = xe + wm * TM * 16 + (lane & 15);
  msk::f32x4_t acc[TN][TM];
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int m = 0; m < TM; ++m) acc[n][m] = msk::f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](int sl, int buf) {
    const unsigned char* sx = ring + buf * SBYTES + wm * TM * kRows16;
    const unsigned char* sw = ring + buf * SBYTES + BM * kBlock + wn * TN * kRows16;
    if constexpr (EIGHT) {
      auto codes = [&](const unsigned char* p) {
        const uint4 lo = *reinterpret_cast<const uint4*>(p + fo[0]), hi = *reinterpret_cast<const uint4*>(p + fo[1]);
        return i32x8_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                       static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
      };
      i32x8_t A[TN];
      int ea[TN];
#pragma unroll
      for (int n = 0; n < TN; ++n) A[n] = codes(sw + n * kRows16), ea[n] = we[wb[n] + sl];
#pragma unroll
      for (int m = 0; m < TM; ++m) {
        const i32x8_t B = codes(sx + m * kRows16);
        const int eb = xel[sl * BM + 16 * m];
#pragma unroll
        for (int n = 0; n < TN; ++n)
          acc[n][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A[n], B, acc[n][m], 0, 0, 0, ea[n], 0, eb);
      }
    } else {
      float sa[TN], sb[TM];
#pragma unroll
      for (int n = 0; n < TN; ++n) sa[n] = scale_of(we[wb[n] + sl]);
#pragma unroll
      for (int m = 0; m < TM; ++m) sb[m] = scale_of(xel[sl * BM + 16 * m]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        msk::bf16x8_t A[TN][2];
#pragma unroll
        for (int n = 0; n < TN; ++n) to_bf16(*reinterpret_cast<const uint4*>(sw + n * kRows16 + fo[h]), sa[n], A[n]);
#pragma unroll
        for (int m = 0; m < TM; ++m) {
          msk::bf16x8_t B[2];
          to_bf16(*reinterpret_cast<const uint4*>(sx + m * kRows16 + fo[h]), sb[m], B);
#pragma unroll
          for (int n = 0; n < TN; ++n) acc[n][m] = msk::mfma16(A[n][0], B[0], acc[n][m]);
#pragma unroll
          for (int n = 0; n < TN; ++n) acc[n][m] = msk::mfma16(A[n][1], B[1], acc[n][m]);
        }
      }
    }
  };
  __syncthreads();  // the exponents are there
  int cur = 0, nxt = NST - 1;
  for (int turn = 0; turn * KS < a.nb; ++turn) {
    msk::wait_vm<(NST - 2) * NL>();
    msk::bare_barrier();
    issue(turn + NST - 1, nxt);
    if (KS == 1 || turn * KS + part < a.nb) compute(turn * KS + part, cur);
    cur = cur + 1 == NST ? 0 : cur + 1;
    nxt = nxt + 1 == NST ? 0 : nxt + 1;
  }
  msk::wait_vm<0>();  // the reloads past the last stage land before the work-group ends, or its LDS is used again
  if constexpr (KS > 1) {  // the parts' sums, in their order
    static_assert((KS - 1) * TN * TM * NWV * 1024 <= KS * NST * SBYTES, "sums");
    auto* sums = reinterpret_cast<msk::f32x4_t*>(lds) + (wv * 64 + lane);
    __syncthreads();
    if (part > 0) {
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m) sums[(((part - 1) * TN + n) * TM + m) * NWV * 64] = acc[n][m];
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 1; p < KS; ++p)
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m) acc[n][m] += sums[(((p - 1) * TN + n) * TM + m) * NWV * 64];
  }
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    const int t = t0 + (wm * TM + m) * 16 + (lane & 15);
    if (t >= a.T) continue;
#pragma unroll
    for (int n = 0; n < TN; ++n) store4<Y>(a, t, o0 + (wn * TN + n) * 16 + 4 * (lane >> 4), acc[n][m], vec);
  }
}

// Prompts: tiles of 256 tokens in eight waves, two to a SIMD, of which one reads a stage's
// operands from LDS while the other's matrix instructions run; they change places at every
// barrier.  Both read a stage: waves 0 .. 3 in phase 2 s, waves 4 .. 7 in phase 2 s + 1, so
// its buffer is loaded again from phase 2 s + 2 on and read from 2 s + 4 on.  A stage's loads
// are spread over what else a wave does in the phase: the CU takes one per 16 cycles, and
// in a row they would hold up what stands behind them.
//   A row of a matrix instruction's block n of outputs, for bf16 results, is one of 32 that
// blocks n and n ^ 1 share, so that a lane ends with eight neighbouring outputs of a token
// and four lanes with 64 bytes in a row (with fp32 results they do as it is): 4096 tokens 128 ->
// 14336, little but results, 51 us without and 37 with it.
//   fp32 results: the tokens' codes become bf16 in the reading phase, the outputs' in the
// multiplying one, a conversion or two behind every matrix instruction (in a row before them
// they cost 84 us for 80 below), and a wave takes 64 x 64 to 64 x 96, which has the fewest
// conversions to a product.
//   Launches after each other on three sets of inputs in turn, so that weights are not in the
// caches: 2048 tokens 4096 -> 6144 fp32 79 us (1.3 PFLOP/s; a library product of bf16 matrices
// 82), bf16 48 (2.1 PFLOP/s; a library product of e4m3 matrices with one scale 46); 4096 tokens
// 4096 -> 14336 370-384 and 222-229 us (1.3 and 2.1 PFLOP/s; 345 and 172); 8192 cubed 813 and
// 435-448 (705 and 356).  On the same inputs again and again the second is 360-371 and 203-212, the
// third 810 and 416-424, and the library's hardly less: the first loads of a tile wait longer here.
//   On the same inputs: of a bf16 stage's 1.3-1.4 us per CU, the matrix instructions alone take 1.2
// and the loads alone 1.1 (15 TB/s from the L2s); a tile's start and end 8 us of 55, the matrix
// cores idle.  Fetching stages ahead into the L2, without waiting for them, made it slower (259 -> 292
// us at the time).
template <bool EIGHT, int BN>
struct Pair {
  static constexpr int BM = 256, WM = EIGHT ? 2 : 4, NWV = 8, WN = NWV / WM;  // tokens, waves
  static constexpr int TN = BN / WN / 16, EW = TN <= 4 ? 4 : 8;               // bytes of a wave's weight exponents
  static constexpr int STAGES = 2 * (BM + BN) * kBlock, WE = 2 * EW * WN * (kMostColumns / kBlock);
};
// The tile of tokens from t0 on and outputs from o0 on, of those before o_stop.
template <typename Y, bool EIGHT, int BN>
__device__ __forceinline__ void dense_q_pair(const DenseArgs& a, int t0, int o0, int o_stop, int vec, unsigned char* lds, uint8_t* xe,
                                             uint8_t* we) {
  using P = Pair<EIGHT, BN>;
  constexpr int BM = P::BM, WM = P::WM, NWV = P::NWV, WN = P::WN;
  constexpr int TM = BM / WM / 16, TN = P::TN, EW = P::EW;
  constexpr int NX = BM / 8 / NWV, NL = (BM + BN) / 8 / NWV;  // loads per wave and stage: tokens', all
  constexpr int SBYTES = (BM + BN) * kBlock;
  static_assert(TM % 4 == 0 && TM <= 8 && TN <= 8 && TN * WN * 16 == BN && BN % (8 * NWV) == 0 && NL <= 8, "tile split");
  static_assert(P::STAGES + kTileExps + P::WE <= 160 * 1024, "LDS");
  constexpr auto paired = [](int n) { return sizeof(Y) == 2 && (n | 1) < TN; };
  const int lane = threadIdx.x & 63, i16 = lane & 15, g4 = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool second = wv >= 4;
  const int wm = wv % WM, wn = wv / WM;
  const uint8_t *x0 = a.x + static_cast<size_t>(t0) * a.n_in, *w0 = a.w + static_cast<size_t>(o0) * a.n_in;

  // Staged rows: the tile's tokens, then its outputs, the last of either again.  Piece p of a
  // token's row r sits in slot p ^ (r % 8), of an output's in that with its halves changed
  // where r / 8 is odd: so the eight rows that are read together have distinct slots in either
  // order.  A load takes eight rows from a uniform address on; lanes' offsets to them are all
  // alike but where the rows end, and from there on.
  const int x_end = min(BM, a.T - t0) - 1, w_end = min(BN, o_stop - o0) - 1;
  const int lrow = lane >> 3, xk = 16 * ((lane & 7) ^ lrow), wk = xk ^ 64 * (wv & 1);
  const uint32_t x_off = lrow * a.n_in + xk, w_off = lrow * a.n_in + wk;
  const uint32_t x_last = min(lrow, x_end % 8) * a.n_in + xk, w_last = min(lrow, w_end % 8) * a.n_in + wk;
  const uint32_t lbase = msk::lds_address(lds) + wv * kStageLoad;
  // Load j of a stage, into the buffer sl % 2; stages past the last reload it (never read).
  // Pieces past a row's end load its first one instead: clear_ends puts zeros in their place.
  auto issue = [&](int sl, int j) {
    const bool x = j < NX;
    const int k0 = min(sl, a.nb - 1) * kBlock, g = wv + NWV * (x ? j : j - NX), last = (x ? x_end : w_end) / 8, k = x ? xk : wk;
    const uint32_t o = g < last ? (x ? x_off : w_off) : (x ? x_last : w_last);
    msk::lds_load16((x ? x0 : w0) + min(g, last) * 8 * a.n_in, o + (k0 + k < a.n_in ? k0 : -k),
                    lbase + (sl & 1) * SBYTES + NWV * j * kStageLoad);
  };
  auto clear_ends = [&](int sl) {  // of the loads of this wave, which have landed
    if (sl != a.nb - 1 || a.n_in % kBlock == 0) return;
#pragma unroll
    for (int j = 0; j < NL; ++j)
      if (sl * kBlock + (j < NX ? xk : wk) >= a.n_in)
        *reinterpret_cast<uint4*>(lds + (sl & 1) * SBYTES + (wv + NWV * j) * kStageLoad + 16 * lane) = make_uint4(0, 0, 0, 0);
  };
#pragma unroll
  for (int j = 0; j < NL; ++j) issue(0, j);
#pragma unroll
  for (int j = 0; j < NL; ++j) issue(1, j);
  stage_exponents<BM, 64 * NWV>(a, t0, [&](int r, int b, uint8_t e) {
    xe[b * BM + (r / (16 * TM) * 16 + r % 16) * TM + r / 16 % TM] = e;
  });
  for (int i = threadIdx.x; i < 2 * EW * WN * a.nb; i += 64 * NWV) {
    const int n = i % EW, half = i / EW % 2, b = i / (2 * EW * WN);
    const int o = min(o0 + (i / (2 * EW) % WN * TN + (paired(n) ? (n & ~1) + half : n)) * 16, a.n_out - 1);
    we[i] = static_cast<uint8_t>(exponent_in_range(a.w_exp[static_cast<size_t>(o / kBlock) * a.nb + b]));
  }
  int xo[2], wo[3][2];  // a lane's pieces of a block of tokens, and of an even, an odd and an unpaired one of outputs
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int piece = 4 * h + g4;
    xo[h] = i16 * kBlock + 16 * (piece ^ (i16 & 7));
#pragma unroll
    for (int n = 0; n < 3; ++n) {
      const int r = n < 2 ? i16 / 4 * 8 + n * 4 + i16 % 4 : i16;
      wo[n][h] = r * kBlock + 16 * (piece ^ (r & 7) ^ (r >> 3 & 1) << 2);
    }
  }

  msk::f32x4_t acc[TN][TM];
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int m = 0; m < TM; ++m) acc[n][m] = msk::f32x4_t{0.f, 0.f, 0.f, 0.f};
  // A stage's operands: codes, or the tokens' in bf16
  uint4 A[TN][2], B[EIGHT ? TM : 1][2];
  msk::bf16x8_t xb[EIGHT ? 1 : TM][2][2];
  uint32_t ea[EW / 4], eb[TM / 4];  // a byte per block of 16 outputs, and of 16 tokens
  auto output_scale = [&](int n) { return ea[n / 4] >> (8 * (n % 4)); };
  auto token_scale = [&](int m) { return eb[m / 4] >> (8 * (m % 4)); };
  msk::bf16x8_t wa[2][2][2];  // two blocks of outputs, the next one made while the last is multiplied
  auto convert = [&](int n) {
#pragma unroll
    for (int h = 0; h < 2; ++h) to_bf16(A[n][h], scale_of(output_scale(n) & 255), wa[n % 2][h]);
  };
  auto read = [&](int sl, auto load) {
    const unsigned char* sx = lds + (sl & 1) * SBYTES + wm * TM * kRows16;
    const unsigned char* sw = lds + (sl & 1) * SBYTES + BM * kBlock + wn * TN * kRows16;
#pragma unroll
    for (int i = 0; i < EW / 4; ++i) ea[i] = *reinterpret_cast<const uint32_t*>(we + ((sl * WN + wn) * 2 + (i16 >> 3)) * EW + 4 * i);
#pragma unroll
    for (int i = 0; i < TM / 4; ++i) eb[i] = *reinterpret_cast<const uint32_t*>(xe + ((sl * WM + wm) * 16 + i16) * TM + 4 * i);
    int j = 0;
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (i >= TM) {
          const int n = i - TM;
          A[n][h] = *reinterpret_cast<const uint4*>(sw + (paired(n) ? n & ~1 : n) * kRows16 + wo[paired(n) ? n & 1 : 2][h]);
          continue;
        }
        const uint4 c = *reinterpret_cast<const uint4*>(sx + i * kRows16 + xo[h]);
        if constexpr (EIGHT)
          B[i][h] = c;
        else
          to_bf16(c, scale_of(token_scale(i) & 255), xb[i][h]);
      }
      while ((i + 1) * NL / (TN + TM) > j) load(j++);
    }
    if constexpr (!EIGHT) convert(0);
  };
  auto pin = []() { __builtin_amdgcn_sched_barrier(0); };
  auto multiply = [&](auto load) {
    int j = 0;
    __builtin_amdgcn_s_setprio(1);
    if constexpr (EIGHT) {
      auto codes = [](const uint4 (&p)[2]) {
        return i32x8_t{static_cast<int>(p[0].x), static_cast<int>(p[0].y), static_cast<int>(p[0].z), static_cast<int>(p[0].w),
                       static_cast<int>(p[1].x), static_cast<int>(p[1].y), static_cast<int>(p[1].z), static_cast<int>(p[1].w)};
      };
#pragma unroll
      for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int n = 0; n < TN; ++n)  // (of a scale the lowest byte counts)
          acc[n][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(A[n]), codes(B[m]), acc[n][m], 0, 0, 0,
                                                                       static_cast<int>(output_scale(n)), 0,
                                                                       static_cast<int>(token_scale(m)));
        while ((m + 1) * NL / TM > j) load(j++);
      }
    } else {
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        if (n + 1 < TN) convert(n + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int m = 0; m < TM; ++m) acc[n][m] = msk::mfma16(wa[n % 2][q / 2][q % 2], xb[m][q / 2][q % 2], acc[n][m]);
        if (n + 1 < TN) {
#pragma unroll
          for (int i = 0; i < 4 * TM; ++i) {  // a conversion behind every matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x2, 2, 0);
          }
        }
        pin();
        while ((n + 1) * NL / TN > j) load(j++);
      }
    }
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int m = 0; m < TM; ++m) asm volatile("" : "+v"(acc[n][m]));  // here, and not behind a barrier or wait
    __builtin_amdgcn_s_setprio(0);
  };
  auto change = [&]() {  // to the next phase
    pin();
    msk::bare_barrier();
    pin();
  };
  msk::wait_vm<0>();
  clear_ends(0);
  clear_ends(1);
  __syncthreads();  // two stages and the exponents are there
  auto none = [](int) {};
  auto turn = [&](int sl, bool first) {  // (stages 0 and 1 are there already: the first turn loads less)
    if (second) {
      read(sl, none);
      msk::wait_vm<0>();
      if (!first) clear_ends(sl + 1);
      change();
      multiply([&](int j) { issue(sl + 2, j); });
    } else {
      read(sl, [&](int j) { if (!first) issue(sl + 1, j); });
      change();
      multiply(none);
      msk::wait_vm<0>();
      if (!first) clear_ends(sl + 1);
    }
    change();
  };
  auto turns = [&]() {  // (the first apart from the loop: 8192 cubed fp32 820 -> 804 us, but bf16 410 -> 445, the same inputs)
    if (!EIGHT) turn(0, true);
    for (int sl = EIGHT ? 0 : 1; sl < a.nb; ++sl) turn(sl, EIGHT && sl == 0);
  };
  if (second) {
    change();
    turns();
  } else {
    turns();
    change();
  }
  msk::wait_vm<0>();  // the reloads past the last stage land before the work-group ends
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    const int t = t0 + (wm * TM + m) * 16 + i16;
    if (t >= a.T) continue;
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const int o = o0 + wn * TN * 16;
      if (!paired(n))
        store4<Y>(a, t, o + n * 16 + 4 * g4, acc[n][m], vec);
      else if (n % 2 == 0)
        store8<Y>(a, t, o + n * 16 + 8 * g4, acc[n][m], acc[n + 1 < TN ? n + 1 : n][m], vec);
    }
  }
}

// Tiles of BN outputs, and of REST from output o_split on in the last `rest` work-groups.
template <typename Y, bool EIGHT, int BN, int REST>
__global__ __launch_bounds__(512, 2) void dense_q_pair_kernel(DenseArgs a, int m_tiles, int vec, int o_split, int rest) {
  __shared__ __align__(16) unsigned char lds[Pair<EIGHT, BN>::STAGES];
  __shared__ __align__(4) uint8_t xe[kTileExps];               // [blocks of columns][WM][16 lanes][TM]
  __shared__ __align__(4) uint8_t we[Pair<EIGHT, BN>::WE];  // [blocks of columns][WN][lanes' halves][EW]
  static_assert(REST <= BN, "LDS");
  const int first = static_cast<int>(gridDim.x) - rest, w = blockIdx.x;
  const bool is_rest = REST != BN && w >= first;
  const int2 tile = is_rest ? tile_of(w - first, rest, m_tiles) : tile_of(w, first, m_tiles);
  // (the divisions are the vector unit's)
  const int t0 = __builtin_amdgcn_readfirstlane(tile.x) * Pair<EIGHT, BN>::BM, at = __builtin_amdgcn_readfirstlane(tile.y);
  if (is_rest)
    dense_q_pair<Y, EIGHT, REST>(a, t0, o_split + at * REST, a.n_out, vec, lds, xe, we);
  else
    dense_q_pair<Y, EIGHT, BN>(a, t0, at * BN, o_split, vec, lds, xe, we);
}

// Tile of a launch: the one whose rounds over the CUs cost least, by the times (0.1 us) of
// one full launch at 4096 columns, fp32 and bf16 results, with one work-group per CU and
// with two, of which the small tiles' overlap.
constexpr int kCus = 256;
struct Tile {
  int bm, bn, parts;   // tokens, outputs; waves that divide the columns
  int one[2], two[2];  // cost of a round
};
constexpr Tile kTiles[] = {{32, 32, 4, {88, 68}, {157, 120}},    {32, 32, 2, {96, 73}, {126, 94}},
                           {64, 64, 4, {141, 106}, {262, 221}},  {64, 64, 2, {155, 107}, {231, 161}},
                           {128, 128, 2, {364, 230}, {691, 439}}, {256, 128, 1, {587, 391}, {1128, 752}},
                           {256, 192, 1, {766, 474}, {1492, 914}}, {256, 256, 1, {0, 562}, {0, 1081}}};
// Whole rounds of one of the two largest tiles, and the outputs that are left in the third: 4096
// tokens 4096 -> 14336 bf16 230 us with the largest alone and 228 with both, 8192 cubed fp32 828 and
// 814, 2048 tokens 4096 -> 14336 fp32 234 and 209 (three sets of inputs in turn).
constexpr int kNTiles = std::size(kTiles), kRest = kNTiles - 3, kFirstMixed = kNTiles - 2;
static_assert(kTiles[kRest].bm == kTiles[kFirstMixed].bm, "the same tokens");

template <typename Y, bool EIGHT>
ms_status launch_tiles(const DenseArgs& a, int vec, hipStream_t s) {
  auto count = [&](const Tile& t, int64_t outputs) {
    return ((static_cast<int64_t>(a.T) + t.bm - 1) / t.bm) * ((outputs + t.bn - 1) / t.bn);
  };
  auto rounds = [&](const Tile& t, int64_t n) {
    const int64_t rest = n % (2 * kCus);
    return n / (2 * kCus) * t.two[EIGHT] + (rest == 0 ? 0 : rest <= kCus ? t.one[EIGHT] : t.two[EIGHT]);
  };
  auto fits = [&](const Tile& t, int64_t n) {  // a launch, and the exponents' LDS
    return n <= UINT32_MAX / 1024 && a.nb * t.bm <= kTileExps;
  };
  int best = -1, o_split = a.n_out;
  int64_t best_cost = INT64_MAX;
  for (int i = 0; i < kNTiles - !EIGHT; ++i) {
    const Tile& t = kTiles[i];
    const int64_t n = count(t, a.n_out);
    if (!fits(t, n)) continue;
    if (const int64_t cost = rounds(t, n); cost < best_cost) best = i, best_cost = cost, o_split = a.n_out;
    // whole rounds of large tiles, and smaller ones for the outputs that are left
    if (i < kFirstMixed || n < kCus) continue;
    const int64_t m = (a.T - 1) / t.bm + 1, wide = n / kCus * kCus / m, left = a.n_out - wide * t.bn;
    if (wide == 0 || left <= 0 || !fits(t, wide * m + count(kTiles[kRest], left))) continue;
    const int64_t cost = rounds(t, wide * m) + rounds(kTiles[kRest], count(kTiles[kRest], left));
    if (cost < best_cost) best = i, best_cost = cost, o_split = static_cast<int>(wide * t.bn);
  }
  if (best < 0) return MS_E_UNSUPPORTED;
  const int m_tiles = (a.T - 1) / kTiles[best].bm + 1;
  const int rest = static_cast<int>(count(kTiles[kRest], a.n_out - o_split));
  const dim3 grid(static_cast<unsigned>(count(kTiles[best], o_split) + rest));
#define MSK_TILE_CASE(I_, BM_, BN_, WM_, WN_, NST_, KS_)                                                                  \
  case I_:                                                                                                                \
    static_assert(kTiles[I_].bm == BM_ && kTiles[I_].bn == BN_ && kTiles[I_].parts == KS_, "tiles");                      \
    hipLaunchKernelGGL((dense_q_tile_kernel<Y, EIGHT, BM_, BN_, WM_, WN_, NST_, KS_>), grid, dim3(64 * WM_ * WN_ * KS_), 0, s, \
                       a, m_tiles, vec);                                                                                  \
    break;
#define MSK_PAIR_CASE(I_, BN_)                                                                                                     \
  case I_:                                                                                                                         \
    static_assert(kTiles[I_].bm == 256 && kTiles[I_].bn == BN_, "tiles");                                                          \
    if constexpr (EIGHT || BN_ < 256) {                                                                                            \
      if (o_split == a.n_out)                                                                                                      \
        hipLaunchKernelGGL((dense_q_pair_kernel<Y, EIGHT, BN_, BN_>), grid, dim3(512), 0, s, a, m_tiles, vec, o_split, 0);    \
      else                                                                                                                         \
        hipLaunchKernelGGL((dense_q_pair_kernel<Y, EIGHT, BN_, 128>), grid, dim3(512), 0, s, a, m_tiles, vec, o_split, rest); \
    }                                                                                                                              \
    break;
  switch (best) {
    MSK_TILE_CASE(0, 32, 32, 2, 2, 3, 4)
    MSK_TILE_CASE(1, 32, 32, 2, 2, 3, 2)
    MSK_TILE_CASE(2, 64, 64, 2, 2, 2, 4)
    MSK_TILE_CASE(3, 64, 64, 2, 2, 2, 2)
    MSK_TILE_CASE(4, 128, 128, 2, 4, 2, 2)
    MSK_PAIR_CASE(5, 128)
    MSK_PAIR_CASE(6, 192)
    MSK_PAIR_CASE(7, 256)
  }
#undef MSK_TILE_CASE
#undef MSK_PAIR_CASE
  return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP;
}

// Blocks of 16 outputs per work-group, and waves.  us with 1 x 8 | 2 x 8 | 2 x 16 | 4 x 4, weights
// not in the caches: one token 4096 -> 4096 5.5 | 6.5 | 6.7 | 10.3 (cached), 4096 -> 6144 8.4 | 7.4 |
// 7.9 | 12.3, 4096 -> 14336 15.1 | 14.3 | 13.3 | 14.5, 4096 -> 32000 30.3 | 26.6 | 24.5 | 29.7, 1024 ->
// 32000 7.6 | 7.6 | 9.6 | 8.2; 16 tokens 4096 -> 6144 12.4 | 9.2 | 9.5 | 13.2, -> 32000 40.0 | 32.0 | 31.0 |
// 31.4.  Long rows of one token want one block and sixteen waves, 8192 -> 8192 14.2 for 18.1
// with 2 x 16, and of 16 tokens not, 21.1 for 18.1.
template <typename Y, int NT>
void launch_few(const DenseArgs& a, int vec, hipStream_t s) {
  const unsigned blocks = (a.n_out - 1) / 16 + 1;
#define MSK_FEW(KW_, MO_)                                                                                              \
  hipLaunchKernelGGL((dense_q_few_kernel<Y, (KW_), (MO_), NT>), dim3((blocks + (MO_) - 1) / (MO_)), dim3(64 * (KW_)), 0, s, \
                     a, vec)
  if (blocks <= kCus) {
    MSK_FEW(8, 1);
  } else if constexpr (NT == 1) {
    if (a.n_in > 4096 && a.T <= 4)
      MSK_FEW(16, 1);
    else if (a.n_in > 4096 || (a.n_in > 2048 && blocks > 2 * kCus))
      MSK_FEW(16, 2);
    else
      MSK_FEW(8, 2);
  } else {
    MSK_FEW(8, 2);
  }
#undef MSK_FEW
}

// Which calls dense_q_few_kernel takes: up to 16 tokens all; up to 32 those of short rows, and of
// longer ones that do not start every 512 bytes on few memory channels (its waves read a row
// in pieces, tiles whole rows); with fp32 results up to 64 those of rows shorter still.  us of
// it | tiles, weights not in the caches: 16 tokens 4096 -> 6144 fp32 8.9 | 8.9, 4096 -> 4096 7.2 |
// 8.7; 32 tokens 2048 -> 4096 fp32 5.9 | 6.7, bf16 5.9 | 6.1, 2048 -> 32000 18.0 | 16.5, 3008 -> 4096 fp32
// 7.0 | 8.6, 4096 -> 4096 10.5 | 9.3; 64 tokens 1520 -> 6144 fp32 8.3 | 8.9, bf16 8.3 | 8.4, 2048 ->
// 6144 fp32 9.8 | 9.0, 4096 -> 4096 (cached) 14.7 | 8.9.
bool takes_few(const DenseArgs& a, bool eight) {
  if (a.T <= 16) return true;
  if (a.n_out > 32 * kCus) return false;
  if (a.T <= 32) return a.n_in <= 2048 || (a.n_in <= 4096 && a.n_in % 512 != 0 && a.n_out <= 16 * kCus);
  return a.T <= 64 && !eight && a.n_in < 2048;
}

template <typename Y, bool EIGHT>
ms_status launch_dense_q(const DenseArgs& a, hipStream_t s) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.add);
  const int vec = a.n_out % 4 == 0 && (at & (4 * sizeof(Y) - 1)) == 0;
  if (!takes_few(a, EIGHT)) return launch_tiles<Y, EIGHT>(a, vec, s);
  if (a.T <= 16)
    launch_few<Y, 1>(a, vec, s);
  else if (a.T <= 32)
    launch_few<Y, 2>(a, vec, s);
  else if constexpr (!EIGHT)
    launch_few<Y, 4>(a, vec, s);
  return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
ms_status launched() { return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP; }
bool value_type(int32_t t) { return t == MS_F32 || t == MS_BF16; }
// rows of 16-byte pieces
ms_status check_columns(int32_t n) {
  if (n <= 0) return MS_E_INVALID;
  return n % 16 == 0 && n <= kMostColumns ? MS_OK : MS_E_UNSUPPORTED;
}
// A row by four waves, a short one by two or one: 4096 rows of 1024 15.4 us with four and
// 12.3 with two, of 256 7.2 with four and 6.7 with one; 4096 rows of 2048 19.7 with four and
// 21.8 with one.
template <typename Y>
void launch_norm(const NormArgs& a, hipStream_t s) {
  const unsigned T = static_cast<unsigned>(a.T);
  const dim3 block(kNormThreads), rows(T), twos((T + 1) / 2), fours((T + 3) / 4);
  const int d = a.d;
#define MSK_NORM(GRID_, WAVES_, PER_) /* (of one wave, rows have no LDS of their own) */ \
  hipLaunchKernelGGL((residual_norm_q_kernel<Y, WAVES_, PER_>), GRID_, block, msk::kGuardLds, s, a)
  if (d <= 512)
    MSK_NORM(fours, 1, 1);
  else if (d <= 1024)
    MSK_NORM(twos, 2, 1);
  else if (d <= 2048)
    MSK_NORM(rows, 4, 1);
  else if (d <= 4096)
    MSK_NORM(rows, 4, 2);
  else if (d <= 8192)
    MSK_NORM(rows, 4, 4);
  else
    MSK_NORM(rows, 4, 8);
#undef MSK_NORM
}

}  // namespace

extern "C" {

ms_status ms_quant_q(const void* x, int32_t dtype, int32_t rows, int32_t n, int32_t block_rows, void* codes, void* exps,
                     void* stream) {
  if (!value_type(dtype) || rows < 0 || (block_rows != 1 && block_rows != kBlock)) return MS_E_INVALID;
  if (const ms_status st = check_columns(n); st != MS_OK) return st;
  if (rows == 0) return MS_OK;
  if (!x || !codes || !exps || !aligned16(x) || !aligned16(codes)) return MS_E_INVALID;
  const int nb = (n + kBlock - 1) / kBlock;
  const size_t values = static_cast<size_t>(rows) * n, ne = (static_cast<size_t>(rows) + block_rows - 1) / block_rows * nb;
  const size_t bytes = values * (dtype == MS_F32 ? 4 : 2);
  if (overlap(codes, values, x, bytes) || overlap(exps, ne, x, bytes) || overlap(codes, values, exps, ne)) return MS_E_INVALID;
  const int64_t wgs = block_rows == 1 ? (static_cast<int64_t>(rows) * nb * 16 + kQuantThreads - 1) / kQuantThreads
                                      : (static_cast<int64_t>(rows) + kBlock - 1) / kBlock * nb;
  if (wgs > UINT32_MAX / kQuantThreads) return MS_E_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(wgs)), block(kQuantThreads);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  auto* c = static_cast<uint8_t*>(codes);
  auto* e = static_cast<uint8_t*>(exps);
  const auto* f = static_cast<const float*>(x);
  const auto* b = static_cast<const uint16_t*>(x);
  if (block_rows == 1 && dtype == MS_F32)
    hipLaunchKernelGGL(quant_rows_kernel<float>, grid, block, msk::kGuardLds, s, f, rows, n, nb, c, e);
  else if (block_rows == 1)
    hipLaunchKernelGGL(quant_rows_kernel<uint16_t>, grid, block, msk::kGuardLds, s, b, rows, n, nb, c, e);
  else if (dtype == MS_F32)
    hipLaunchKernelGGL(quant_blocks_kernel<float>, grid, block, 0, s, f, rows, n, nb, c, e);
  else
    hipLaunchKernelGGL(quant_blocks_kernel<uint16_t>, grid, block, 0, s, b, rows, n, nb, c, e);
  return launched();
}

ms_status ms_residual_norm_q(const void* h, const void* y, int32_t y_dtype, const void* weight, double eps, int32_t T,
                             int32_t d, void* sum_out, void* out, void* codes, void* exps, void* stream) {
  if (!value_type(y_dtype) || T < 0 || !(eps >= 0.0) || !std::isfinite(eps)) return MS_E_INVALID;
  if (const ms_status st = check_columns(d); st != MS_OK) return st;
  if (T == 0) return MS_OK;
  if (!h || (!sum_out && !out && !codes) || !codes != !exps) return MS_E_INVALID;
  if (!aligned16(h) || !aligned16(y) || !aligned16(weight) || !aligned16(sum_out) || !aligned16(out) || !aligned16(codes))
    return MS_E_INVALID;
  // a row is read whole before any of it is written, and by nobody else: sum_out or out may be h or a bf16 y
  const size_t n = static_cast<size_t>(T) * d, ny = n * (y_dtype == MS_F32 ? 4 : 2);
  auto clash = [&](const void* o, size_t bytes) {
    return (o != h && overlap(o, bytes, h, 2 * n)) || (!(o == y && ny == 2 * n) && overlap(o, bytes, y, ny)) ||
           overlap(o, bytes, weight, 2 * static_cast<size_t>(d));
  };
  if (clash(sum_out, 2 * n) || clash(out, 2 * n) || overlap(sum_out, 2 * n, out, 2 * n)) return MS_E_INVALID;
  const size_t nb = (d + kBlock - 1) / kBlock, ne = static_cast<size_t>(T) * nb;
  auto apart = [&](const void* o, size_t bytes) {  // codes and exponents: from everything
    return !overlap(o, bytes, h, 2 * n) && !overlap(o, bytes, y, ny) && !overlap(o, bytes, weight, 2 * static_cast<size_t>(d)) &&
           !overlap(o, bytes, sum_out, 2 * n) && !overlap(o, bytes, out, 2 * n);
  };
  if (!apart(codes, n) || !apart(exps, ne) || overlap(codes, n, exps, ne)) return MS_E_INVALID;
  NormArgs a;
  a.h = static_cast<const uint16_t*>(h);
  a.y = y;
  a.weight = static_cast<const uint16_t*>(weight);
  a.sum_out = static_cast<uint16_t*>(sum_out);
  a.out = static_cast<uint16_t*>(out);
  a.codes = static_cast<uint8_t*>(codes);
  a.exps = static_cast<uint8_t*>(exps);
  a.eps = eps;
  a.T = T;
  a.d = d;
  a.nb = static_cast<int>(nb);
  if (T > kMostRows - 1) return MS_E_UNSUPPORTED;
  if (y_dtype == MS_F32)
    launch_norm<float>(a, static_cast<hipStream_t>(stream));
  else
    launch_norm<uint16_t>(a, static_cast<hipStream_t>(stream));
  return launched();
}

ms_status ms_dense_q(const void* x, const void* x_exp, const void* w, const void* w_exp, int32_t T, int32_t n_in,
                     int32_t n_out, void* y, int32_t y_dtype, const void* add, void* stream) {
  if (!value_type(y_dtype) || T < 0 || n_out <= 0) return MS_E_INVALID;
  if (const ms_status st = check_columns(n_in); st != MS_OK) return st;
  if (T == 0) return MS_OK;
  if (!x || !x_exp || !w || !w_exp || !y || !aligned16(x) || !aligned16(w)) return MS_E_INVALID;
  const size_t nb = (n_in + kBlock - 1) / kBlock, rows = T, outs = n_out;
  const size_t bytes = rows * outs * (y_dtype == MS_F32 ? 4 : 2);
  if (overlap(y, bytes, x, rows * n_in) || overlap(y, bytes, w, outs * n_in) || overlap(y, bytes, x_exp, rows * nb) ||
      overlap(y, bytes, w_exp, (outs + kBlock - 1) / kBlock * nb) || (add != y && overlap(y, bytes, add, bytes)))
    return MS_E_INVALID;
  const DenseArgs a = {static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(x_exp), static_cast<const uint8_t*>(w),
                       static_cast<const uint8_t*>(w_exp), add, y, T, n_in, n_out, static_cast<int>(nb)};
  if (n_out > kMostOutputs) return MS_E_UNSUPPORTED;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return y_dtype == MS_F32 ? launch_dense_q<float, false>(a, s) : launch_dense_q<uint16_t, true>(a, s);
}

}  // extern "C"
