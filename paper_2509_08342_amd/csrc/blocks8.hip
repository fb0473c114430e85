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

#include "device.h"
#include "kernels.h"
#include "moesplit.h"

namespace {

constexpr int kBlock = 128;  // columns that share a scale, and rows of a weight's block
constexpr int kExpBias = 127;
constexpr int kExpMin = -40, kExpMax = 40;
constexpr float kCodeMax = 448.0f;
constexpr int kMostColumns = 16384;

__device__ __forceinline__ uint32_t bf16_bits(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));  // to nearest even, NaN stays NaN
}

// 2^e, e in [-126, 127]
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
__device__ __forceinline__ double pow2_64(int e) {
  return __longlong_as_double(static_cast<long long>(e + 1023) << 52);
}

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
// Sixteen lanes take 128 columns of a row, eight values each.  ROWS = 1: a block is theirs.
// ROWS = 128: a work-group takes a block, its values in registers until its largest
// magnitude is known.
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
// A work-group per row, sixteen lanes to 128 columns.  The sum of squares, the norm and the
// choice of a block's exponent are in double precision (a code is the nearest to the exact
// normalised value, and no exponent depends on how fp32 would have rounded next to a power
// of two); h and y stay in registers between the two uses.
constexpr int kNormThreads = 256;

// d as fp32 that a second rounding, to bf16 or a code, cannot tell from d: of the two
// neighbours the one with an odd last bit where d is neither.
__device__ __forceinline__ float to_odd(double d) {
  const float f = static_cast<float>(d);
  const double e = d - f;
  const uint32_t u = __float_as_uint(f);
  if (!(e > 0.0 || e < 0.0) || (u & 1)) return f;  // exact, or not finite, or odd
  return __uint_as_float((e > 0.0) == (u >> 31 == 0) ? u + 1 : u - 1);
}

// the least fp32 that is not below |d|, 0 for what is not finite
__device__ __forceinline__ uint32_t magnitude_up(double d) {
  const double a = fabs(d);
  if (!(a < INFINITY)) return 0;
  const float f = static_cast<float>(a);
  if (!(f < INFINITY)) return 0x7f7fffffu;
  return __float_as_uint(f) + (static_cast<double>(f) < a);
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
  int d, nb;
};

template <typename Y, int PER>
__global__ __launch_bounds__(kNormThreads) void residual_norm_q_kernel(NormArgs a) {
  __shared__ double sums[kNormThreads / 64];
  const size_t row = static_cast<size_t>(blockIdx.x) * a.d;
  const Y* y = static_cast<const Y*>(a.y);
  float h[PER][8], r[PER][8];
  double ss = 0.0;
#pragma unroll
  for (int m = 0; m < PER; ++m) {
    const int k = 8 * (static_cast<int>(threadIdx.x) + m * kNormThreads);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[m][i] = r[m][i] = 0.0f;
    if (k < a.d) {
      load8(a.h + row + k, h[m]);
      if (y) load8(y + row + k, r[m]);
    }
  }
#pragma unroll
  for (int m = 0; m < PER; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double x = static_cast<double>(h[m][i]) + r[m][i];
      ss = fma(x, x, ss);
    }
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) ss += __shfl_xor(ss, s, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = ss;
  __syncthreads();
  ss = 0.0;
#pragma unroll
  for (int w = 0; w < kNormThreads / 64; ++w) ss += sums[w];
  const double inv = 1.0 / sqrt(ss / a.d + a.eps);
#pragma unroll
  for (int m = 0; m < PER; ++m) {
    const int piece = threadIdx.x + m * kNormThreads, k = 8 * piece;
    const bool in = k < a.d;
    double v[8];
    float g[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 1.0f;
    if (in && a.weight) load8(a.weight + k, g);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = static_cast<double>(h[m][i]) + r[m][i];
      f[i] = to_odd(v[i]);
      v[i] *= inv * g[i];
    }
    if (in && a.sum_out) *reinterpret_cast<uint4*>(a.sum_out + row + k) = pack_bf16(f);
    if (in && a.out) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_odd(v[i]);
      *reinterpret_cast<uint4*>(a.out + row + k) = pack_bf16(f);
    }
    if (a.codes) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, in ? magnitude_up(v[i]) : 0u);
      const int e = block_exponent(max_of_lanes(top, 16));
      const double scale = pow2_64(-e);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_odd(fmin(fmax(v[i], -1e30), 1e30) * scale);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = fabs(v[i]) < INFINITY ? f[i] : NAN;
      if (in) {
        *reinterpret_cast<uint2*>(a.codes + row + k) = codes8(f);
        if ((threadIdx.x & 15) == 0)
          a.exps[static_cast<size_t>(blockIdx.x) * a.nb + piece / 16] = static_cast<uint8_t>(e + kExpBias);
      }
    }
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

__device__ __forceinline__ float stored_scale(uint8_t e) {
  return pow2(min(max(static_cast<int>(e) - kExpBias, kExpMin), kExpMax));
}

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(uint16_t* p, float v) { *p = static_cast<uint16_t>(bf16_bits(v)); }

// y^T = W x^T, a wave per 16 outputs x 16 tokens: lane l has sixteen codes of row l % 16 at
// k + 16 (l / 16).
template <typename Y>
__global__ __launch_bounds__(64) void dense_q_simple_kernel(DenseArgs a) {
  const int lane = threadIdx.x, t = blockIdx.x * 16 + (lane & 15), o0 = blockIdx.y * 16, o = o0 + (lane & 15);
  const int tr = min(t, a.T - 1), orow = min(o, a.n_out - 1);
  msk::f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < a.n_in; k0 += 64) {
    const int k = k0 + 16 * (lane >> 4), kb = k0 / kBlock;
    uint4 cx = make_uint4(0, 0, 0, 0), cw = cx;
    if (k < a.n_in) {
      cx = *reinterpret_cast<const uint4*>(a.x + static_cast<size_t>(tr) * a.n_in + k);
      cw = *reinterpret_cast<const uint4*>(a.w + static_cast<size_t>(orow) * a.n_in + k);
    }
    msk::bf16x8_t A[2], B[2];
    to_bf16(cw, stored_scale(a.w_exp[static_cast<size_t>(orow / kBlock) * a.nb + kb]), A);
    to_bf16(cx, stored_scale(a.x_exp[static_cast<size_t>(tr) * a.nb + kb]), B);
    acc = msk::mfma16(A[0], B[0], acc);
    acc = msk::mfma16(A[1], B[1], acc);
  }
  if (t >= a.T) return;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int c = o0 + 4 * (lane >> 4) + r;
    if (c >= a.n_out) continue;
    const size_t i = static_cast<size_t>(t) * a.n_out + c;
    const float add = a.add ? load_value(static_cast<const Y*>(a.add)[i]) : 0.0f;
    store_value(static_cast<Y*>(a.y) + i, acc[r] + add);
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
ms_status launched() { return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP; }
bool value_type(int32_t t) { return t == MS_F32 || t == MS_BF16; }
// rows of 16-byte pieces
ms_status check_columns(int32_t n) {
  if (n <= 0) return MS_E_INVALID;
  return n % 16 == 0 && n <= kMostColumns ? MS_OK : MS_E_UNSUPPORTED;
}
bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const auto a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && a < b + nq && b < a + np;
}

template <typename Y>
void launch_norm(const NormArgs& a, int T, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(T)), block(kNormThreads);
  const int per = (a.d + 8 * kNormThreads - 1) / (8 * kNormThreads);
  if (per <= 1)
    hipLaunchKernelGGL((residual_norm_q_kernel<Y, 1>), grid, block, 0, s, a);
  else if (per <= 2)
    hipLaunchKernelGGL((residual_norm_q_kernel<Y, 2>), grid, block, 0, s, a);
  else if (per <= 4)
    hipLaunchKernelGGL((residual_norm_q_kernel<Y, 4>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((residual_norm_q_kernel<Y, 8>), grid, block, 0, s, a);
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
  a.d = d;
  a.nb = static_cast<int>(nb);
  if (y_dtype == MS_F32)
    launch_norm<float>(a, T, static_cast<hipStream_t>(stream));
  else
    launch_norm<uint16_t>(a, T, static_cast<hipStream_t>(stream));
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
  const int64_t tiles = (static_cast<int64_t>(n_out) + 15) / 16;
  if (tiles > 65535 * int64_t{64}) return MS_E_UNSUPPORTED;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((T + 15) / 16, static_cast<unsigned>(tiles));
  if (y_dtype == MS_F32)
    hipLaunchKernelGGL(dense_q_simple_kernel<float>, grid, dim3(64), msk::kGuardLds, s, a);
  else
    hipLaunchKernelGGL(dense_q_simple_kernel<uint16_t>, grid, dim3(64), msk::kGuardLds, s, a);
  return launched();
}

}  // extern "C"
