// Kernels of the 8-bit key/value cache: rotary embedding with the quantising
// append, the cache read back, and grouped-query attention over it with masks,
// capped scores and distance bias, for batches of sequences and contexts of any
// length.  Stateless entry points: every buffer is the caller's, every call is
// enqueued on the caller's stream.
//
// A value is an e4m3 code times a power of two that 64 positions of a head
// share.  A power of two, because the matrix-core operands are made from codes
// by conversions that take the code alone (bf16 and fp16 hold every e4m3 value
// exactly): a key's scale multiplies its score, a value's scale the
// probability, both exact; and raising the scale of positions already there
// moves codes by whole steps.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "device.h"
#include "kernels.h"
#include "moesplit.h"

namespace {

constexpr int kKvBlock = 64;     // positions that share a scale, and keys of an attention tile
constexpr int kExpBias = 127;    // of a stored exponent
constexpr int kExpMin = -40, kExpMax = 40;
constexpr float kCodeMax = 448.0f;
constexpr float kLog2e = 1.4426950408889634f;

typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));  // to nearest even, NaN stays NaN
}

// 2^e, e in [-126, 127]
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// a stored exponent, kept in range whatever the byte holds
__device__ __forceinline__ int exponent(uint8_t x) { return min(max(static_cast<int>(x) - kExpBias, kExpMin), kExpMax); }

// four codes -> fp32
__device__ __forceinline__ void decode4(uint32_t c, float (&v)[4]) {
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), false);
  const f32x2_t b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), true);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
}

// the value to convert: within the codes' range, NaN for what is not finite
__device__ __forceinline__ float code_range(float x) {
  return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? fminf(fmaxf(x, -kCodeMax), kCodeMax) : __uint_as_float(0x7fc00000u);
}

__device__ __forceinline__ uint32_t encode4(const float (&v)[4], float scale) {
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = code_range(v[i] * scale);
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  c = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c, true);
  return static_cast<uint32_t>(c);
}

// Tokens of sequence s: first position and count, 0 if it is not in use.
struct Span {
  int start, count;
};
__device__ __forceinline__ Span span_of(const int32_t* span, int s, int pos0, int T) {
  if (!span) return {pos0, T};
  const int a = span[2 * s], n = span[2 * s + 1];
  return a >= 0 && a <= pos0 && n >= 1 && n <= T ? Span{a, n} : Span{0, 0};
}

// ------------------------------------------------------ rotary and append
//
// Work-group: the tokens of one sequence that fall into one block of 64 cache
// positions, for `group` heads or fewer one after another (queries, keys and values alike).
// The tokens' angles are computed once (LDS), reduced to a fraction of a turn in
// double precision.  Thread c of a row takes four consecutive values; a key's
// or value's stay in registers between the block's largest magnitude and their codes.
// 2048 tokens of 48 heads of 128, 71 MB, take 22 us (3.2 TB/s), a token of them 5.1: the
// bytes, and the double precision of keys, whose registers leave two waves a SIMD.  In
// fp32 alone they took 20 and 4.6, and a few keys in a million got the code beside the
// nearest one.
constexpr int append_threads(int D) { return D == 256 ? 512 : 256; }  // at most 8 passes of a row's threads over 64
constexpr int kAppendGroups = 512;  // the work-groups that a call is cut into by heads

struct AppendArgs {
  const float* qkv;
  uint16_t* q_out;
  uint8_t *k, *v, *k_exp, *v_exp;
  const int32_t* span;
  int T, Hq, Hkv, max_ctx, pos0, blocks, group;
  int rot, interleaved;
  double log2_base, inv_factor, turns, low, inv_ramp, mscale;  // turns: orig_ctx / 2 pi, 0 for f / factor
};

// turns per position of pair i
__device__ __forceinline__ double pair_turns(const AppendArgs& a, int i) {
  const double f = exp2(-2.0 * i / a.rot * a.log2_base);
  double keep = 0.0;
  if (a.turns > 0.0) keep = fmin(fmax((a.turns * f - a.low) * a.inv_ramp, 0.0), 1.0);
  return f * ((1.0 - keep) * a.inv_factor + keep) * 0.15915494309189535;
}

// Cosine and sine of t turns times scale: the rest x to a quarter, in half turns, |x| <=
// 1/4, and the series of both there, to 2^-33.
__device__ __forceinline__ double2 turn_of(double t, double scale) {
  const double q = rint(4.0 * t), x = fma(-0.5, q, 2.0 * t), y = x * x;
  double s = -0.007370430945714348, c = -0.02580689139001405;
  s = fma(s, y, 0.08214588661112819);
  s = fma(s, y, -0.5992645293207919);
  s = fma(s, y, 2.550164039877345);
  s = fma(s, y, -5.167712780049969);
  s = fma(s, y, 3.141592653589793) * x * scale;
  c = fma(c, y, 0.23533063035889312);
  c = fma(c, y, -1.3352627688545893);
  c = fma(c, y, 4.058712126416768);
  c = fma(c, y, -4.934802200544679);
  c = fma(c, y, 1.0) * scale;
  const int n = static_cast<int>(q - 4.0 * floor(0.25 * q));
  const double a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_double2(n == 1 || n == 2 ? -a : a, n >= 2 ? -b : b);
}

// d as fp32 that a second rounding, to a code, cannot tell from d: of the two neighbours
// the one with an odd last bit where d is neither.
__device__ __forceinline__ float to_odd(double d) {
  const float f = static_cast<float>(d);
  const double e = d - f;
  const uint32_t u = __float_as_uint(f);
  if (!(e > 0.0 || e < 0.0) || (u & 1)) return f;  // exact, or not finite, or odd
  return __uint_as_float((e > 0.0) == (u >> 31 == 0) ? u + 1 : u - 1);
}

// One value of a turned pair: u c + w s, *t = (c, s), *rest what their rounding to fp32
// left.  Keys in double precision (exact: a key's code is the nearest to the turned value,
// not to its rounding to fp32), queries in fp32, as they go on as bf16, from the same
// angles: a token's query does not depend on how its call is cut up.
template <bool KEY>
__device__ __forceinline__ float turned(float u, float w, const float2* t, const float2* rest) {
  const float2 c = *t;
  if constexpr (!KEY) return fmaf(u, c.x, w * c.y);
  const float2 r = *rest;
  return to_odd(u * (static_cast<double>(c.x) + r.x) + w * (static_cast<double>(c.y) + r.y));
}

template <int D>
__global__ __launch_bounds__(append_threads(D)) void rope_kv_q_kernel(AppendArgs a) {
  constexpr int THREADS = append_threads(D), COLS = D / 4, ROWS = THREADS / COLS, PASSES = kKvBlock / ROWS;
  extern __shared__ __align__(16) float2 turn_s[];  // [tokens][rot / 2] cosine and sine, then what their rounding left
  __shared__ uint32_t top_s[2][THREADS / 64];
  const int heads = a.Hq + 2 * a.Hkv, groups = (heads + a.group - 1) / a.group;
  const int b = blockIdx.x % a.blocks, hg = blockIdx.x / a.blocks % groups, seq = blockIdx.x / a.blocks / groups;
  const Span sp = span_of(a.span, seq, a.pos0, a.T);
  const int base = (sp.start / kKvBlock + b) * kKvBlock;
  const int lo = max(sp.start, base), hi = min(sp.start + sp.count, base + kKvBlock);
  if (lo >= hi) return;  // uniform
  const int c4 = threadIdx.x % COLS, r0 = threadIdx.x / COLS, j0 = 4 * c4, half = a.rot / 2;
  const size_t pitch = static_cast<size_t>(heads) * D;
  const float* src = a.qkv + (static_cast<size_t>(seq) * a.T + (lo - sp.start)) * pitch + j0;  // of token lo
  // a pair's partners of this thread's values: the next value, or `half` away
  const bool turns = j0 < a.rot, vec = half % 4 == 0, first4 = j0 < half;
  const int partner = (threadIdx.x & 63) + (first4 ? half / 4 : -(half / 4));  // of the same row

  float2* const rest_s = turn_s + min(a.T, kKvBlock) * half;
  if (half > 0 && hg < a.Hq + a.Hkv) {  // (its heads are hg, hg + groups, ...: keys, which take longest, are spread)
    int lanes = 1;  // pairs side by side: a power of two
    while (lanes < half) lanes *= 2;
    const int i = threadIdx.x % lanes;
    if (i < half) {
      const double f = pair_turns(a, i);
      for (int p = lo + static_cast<int>(threadIdx.x) / lanes; p < hi; p += THREADS / lanes) {
        const double2 t = turn_of(p * f, a.mscale);
        const float2 near = make_float2(static_cast<float>(t.x), static_cast<float>(t.y));
        const int at = (p - lo) * half + i;
        turn_s[at] = near;
        rest_s[at] = make_float2(static_cast<float>(t.x - near.x), static_cast<float>(t.y - near.y));
      }
    }
  }
  __syncthreads();

  for (int head = hg, nth = 0; head < heads; head += groups, ++nth) {
    const bool turn = turns && head < a.Hq + a.Hkv, value = head >= a.Hq + a.Hkv, key = head >= a.Hq;
    const size_t row = static_cast<size_t>(seq) * a.Hkv + (value ? head - a.Hq - a.Hkv : head - a.Hq);  // keys and values
    uint8_t* exps = (value ? a.v_exp : a.k_exp) + row * (a.max_ctx / kKvBlock) + base / kKvBlock;
    const int was = head >= a.Hq && lo > base ? exponent(*exps) : kExpMin;
    const float* x = src + static_cast<size_t>(head) * D;
    float val[PASSES][4];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int p = lo + i * ROWS + r0;
      float4 own = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p < hi) own = *reinterpret_cast<const float4*>(x + static_cast<size_t>(p - lo) * pitch);
      val[i][0] = own.x, val[i][1] = own.y, val[i][2] = own.z, val[i][3] = own.w;
    }
    auto rotate = [&](auto is_key) {
      constexpr bool KEY = decltype(is_key)::value;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int p = lo + i * ROWS + r0;
        if (p >= hi) continue;  // a row's threads alike
        const float2 *cs = turn_s + (p - lo) * half, *rest = rest_s + (p - lo) * half;
        const float* xr = x + static_cast<size_t>(p - lo) * pitch;
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const int m = (j0 + e) / 2;
            if (j0 + e >= a.rot) continue;
            const float u = val[i][e], w = val[i][e + 1];
            val[i][e] = turned<KEY>(u, -w, cs + m, rest + m);
            val[i][e + 1] = turned<KEY>(w, u, cs + m, rest + m);
          }
        } else if (vec) {  // the four values are on one side
          float other[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) other[e] = __shfl(val[i][e], partner, 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int m = first4 ? j0 + e : j0 + e - half;
            val[i][e] = turned<KEY>(val[i][e], first4 ? -other[e] : other[e], cs + m, rest + m);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + e, m = j < half ? j : j - half;
            if (j >= a.rot) continue;
            val[i][e] = turned<KEY>(val[i][e], j < half ? -xr[e + half] : xr[e - half], cs + m, rest + m);
          }
        }
      }
    };
    if (turn && key)
      rotate(std::true_type{});
    else if (turn)
      rotate(std::false_type{});
    if (head < a.Hq) {
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int p = lo + i * ROWS + r0;
        if (p < hi)
          *reinterpret_cast<uint2*>(a.q_out + ((static_cast<size_t>(seq) * a.T + (p - sp.start)) * a.Hq + head) * D + j0) =
              make_uint2(f32_to_bf16_bits(val[i][0]) | f32_to_bf16_bits(val[i][1]) << 16,
                         f32_to_bf16_bits(val[i][2]) | f32_to_bf16_bits(val[i][3]) << 16);
      }
      continue;
    }
    uint32_t top = 0;  // bits of the largest finite magnitude
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t u = __float_as_uint(val[i][e]) & 0x7fffffffu;
        if (u < 0x7f800000u) top = max(top, u);
      }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), s, 64)));
    uint32_t* tops = top_s[nth & 1];  // two in turn: the last head's are read before the barrier of this one's
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();  // every thread has read the old exponent too
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, tops[w]);
    // top = m 2^x, 1 <= m < 2, and 448 = 1.75 * 2^8; zero and subnormal magnitudes end at kExpMin
    int ex = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
    ex = max(min(max(ex, kExpMin), kExpMax), was);
    if (threadIdx.x == 0) *exps = static_cast<uint8_t>(ex + kExpBias);
    uint8_t* out = (value ? a.v : a.k) + (row * a.max_ctx + base) * D;
    const float scale = pow2(-ex);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int p = lo + i * ROWS + r0;
      if (p < hi) *reinterpret_cast<uint32_t*>(out + static_cast<size_t>(p - base) * D + j0) = encode4(val[i], scale);
    }
    if (lo > base && ex > was) {  // the positions before the append, at the new exponent
      const float down = pow2(was - ex);
      for (int i = threadIdx.x; i < (lo - base) * COLS; i += THREADS) {
        uint32_t* w = reinterpret_cast<uint32_t*>(out) + i;
        float v[4];
        decode4(*w, v);
        *w = encode4(v, down);
      }
    }
  }
}

// ------------------------------------------------------------- read back
//
// 16 codes per thread.  Half its start and end, half its bytes: 2048 positions of 8 heads
// of 128 (12.6 MB, 2.7 us at a copy's rate) take 4.8 to 5.5 us, one position 2.6.
constexpr int kReadThreads = 256;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint2 codes_to_bf16(uint32_t c, float scale) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(c), scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(c), scale, true)));
}

__global__ __launch_bounds__(kReadThreads) void kv_read_q_kernel(const uint8_t* __restrict__ k, const uint8_t* __restrict__ v,
                                                                 const uint8_t* __restrict__ k_exp,
                                                                 const uint8_t* __restrict__ v_exp, int D, int max_ctx,
                                                                 int pos0, int n, int per_head, uint16_t* __restrict__ k_out,
                                                                 uint16_t* __restrict__ v_out) {
  const int row = blockIdx.x / per_head;  // sequence and head
  const int64_t i = static_cast<int64_t>(blockIdx.x % per_head) * kReadThreads + threadIdx.x;
  const int pieces = D / 16;
  if (i >= static_cast<int64_t>(n) * pieces) return;
  const int p = pos0 + static_cast<int>(i / pieces);
  const size_t at = (static_cast<size_t>(row) * max_ctx + pos0) * D + 16 * static_cast<size_t>(i);
  const size_t to = static_cast<size_t>(row) * n * D + 16 * static_cast<size_t>(i);
  const size_t ei = static_cast<size_t>(row) * (max_ctx / kKvBlock) + p / kKvBlock;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const uint4 c = *reinterpret_cast<const uint4*>((w ? v : k) + at);
    const float s = pow2(exponent((w ? v_exp : k_exp)[ei]));
    const uint2 a = codes_to_bf16(c.x, s), b = codes_to_bf16(c.y, s), d = codes_to_bf16(c.z, s), e = codes_to_bf16(c.w, s);
    uint4* o = reinterpret_cast<uint4*>((w ? v_out : k_out) + to);
    o[0] = make_uint4(a.x, a.y, b.x, b.y);
    o[1] = make_uint4(d.x, d.y, e.x, e.y);
  }
}

// --------------------------------------------------------------- attention

struct AttArgs {
  const uint16_t* q;
  const uint8_t *k, *v, *k_exp, *v_exp;
  const int32_t* span;
  const float* slopes;
  const int32_t* docs;
  uint16_t* out;
  float* part;  // splits > 1: [rows][splits][D] results of a share of the keys
  float2* ml;   // [rows][splits] the exponent that their sums are relative to (-inf: no key), and the sums
  int T, Hq, Hkv, G, max_ctx, pos0;
  int heads, splits, share;  // key/value heads of all sequences, shares of a row's tiles, and tiles of a share (few rows)
  int window, prefix;
  int scores;           // whether scores are capped or biased
  float pre, cap, mul;  // score = pre q.k, capped and biased; weight = 2^(mul (score - maximum))
};

// Tiles of 64 keys that queries at positions p0 .. p1 of a sequence of n keys
// may see: [0, pre), the prefix, then [lo, hi).
struct Tiles {
  int pre, lo, hi;
  __device__ int count() const { return pre + hi - lo; }
  __device__ int at(int i) const { return i < pre ? i : lo + i - pre; }
};
__device__ __forceinline__ Tiles tiles_of(const AttArgs& a, int p0, int p1, int n) {
  Tiles t;
  const int pre = (min(a.prefix, n) + kKvBlock - 1) / kKvBlock;
  t.lo = a.window > 0 ? max(p0 - a.window + 1, 0) / kKvBlock : 0;
  t.hi = max(p1 / kKvBlock + 1, pre);
  t.pre = min(pre, t.lo);
  return t;
}

// tanh, off by less than 2^-20 of itself.  Up to kSeries in size its series, off by 2^-22;
// above, where 1 - e does not cancel, the exponential's form.
constexpr float kSeries = 0.25f;
__device__ __forceinline__ float tanh_series(float x) {
  const float y = x * x;
  return x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
}
__device__ __forceinline__ float tanh_of(float x) {
  const float e = __builtin_amdgcn_exp2f(fabsf(x) * (-2.0f * kLog2e));
  const float far = (1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e);
  return fabsf(x) < kSeries ? tanh_series(x) : copysignf(far, x);
}

// Whether the query at position i sees key j of n (document di, dj).
__device__ __forceinline__ bool sees(const AttArgs& a, int i, int j, int n, int di, int dj) {
  const int d = i - j;
  bool s = (d >= 0 && (a.window <= 0 || d < a.window)) || j < a.prefix;
  s = s && j < n;
  if (a.docs) s = s && di == dj && di >= 0;
  return s;
}

__device__ __forceinline__ size_t kv_row(const AttArgs& a, int head) { return static_cast<size_t>(head) * a.max_ctx; }
__device__ __forceinline__ size_t exp_row(const AttArgs& a, int head) {
  return static_cast<size_t>(head) * (a.max_ctx / kKvBlock);
}
// row r (token r / G, query head r % G of the group) of a key/value head: its place in q and out, and in part
__device__ __forceinline__ size_t q_row(const AttArgs& a, int head, int r) {
  return (static_cast<size_t>(head / a.Hkv) * a.T + r / a.G) * a.Hq + head % a.Hkv * a.G + r % a.G;
}
__device__ __forceinline__ size_t part_row(const AttArgs& a, int head, int r, int z) {
  return (static_cast<size_t>(head) * a.T * a.G + r) * a.splits + z;
}

// The scales' exponents of 64 list places of a share [i0, i1), one per lane: read
// in the loop by lane, so that no load of theirs makes the loop wait for others.
struct Exps {
  int chunk = -1, both = 0;
  __device__ __forceinline__ void at(const Tiles& tl, int i0, int i1, int i, const uint8_t* ke, const uint8_t* ve, int& ek,
                                     int& ev) {
    const int d = i - i0;
    if (d / 64 != chunk) {
      chunk = d / 64;
      const int tile = tl.at(min(i0 + 64 * chunk + static_cast<int>(threadIdx.x & 63), i1 - 1));
      both = exponent(ke[tile]) << 16 | (exponent(ve[tile]) & 0xffff);
    }
    const int x = __builtin_amdgcn_readlane(both, d & 63);
    ek = x >> 16;
    ev = static_cast<int16_t>(x);
  }
};

// One query row over the tiles [i0, i1) of `tl`, by one wave: lane j of a tile
// has key j's score, then D / 64 columns of the output.  Reads no value that
// the row does not see, so it is what a work-group falls back to when a result
// is not finite (qs: D floats of LDS of the wave's own).
template <int D>
__device__ __forceinline__ void attend_row(const AttArgs& a, int head, const Span& sp, int r, const Tiles& tl, int i0, int i1,
                                           int z, float* qs) {
  constexpr int CPL = D / 64;
  const int lane = threadIdx.x & 63;
  const int pos = sp.start + r / a.G, n = sp.start + sp.count, seq = head / a.Hkv;
  const size_t row = q_row(a, head, r);
#pragma unroll
  for (int c = 0; c < CPL; ++c) qs[CPL * lane + c] = __uint_as_float(static_cast<uint32_t>(a.q[row * D + CPL * lane + c]) << 16);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own row
  const uint8_t *K = a.k + kv_row(a, head) * D, *V = a.v + kv_row(a, head) * D;
  const uint8_t *ke = a.k_exp + exp_row(a, head), *ve = a.v_exp + exp_row(a, head);
  const int32_t* docs = a.docs ? a.docs + static_cast<size_t>(seq) * a.max_ctx : nullptr;
  const int di = docs ? docs[pos] : 0;
  const float slope = a.slopes ? a.slopes[head % a.Hkv * a.G + r % a.G] : 0.0f;
  float m = -INFINITY, l = 0.0f, o[CPL] = {};
  for (int i = i0; i < i1; ++i) {
    const int tile = tl.at(i), j = tile * kKvBlock + lane;
    const bool see = sees(a, pos, j, n, di, docs ? docs[j] : 0);
    float s = -INFINITY;
    if (see) {
      float d = 0.0f;
      for (int c = 0; c < D; c += 16) {
        const uint4 w = *reinterpret_cast<const uint4*>(K + static_cast<size_t>(j) * D + c);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[4];
          decode4(ws[e], v);
#pragma unroll
          for (int f = 0; f < 4; ++f) d = fmaf(qs[c + 4 * e + f], v[f], d);
        }
      }
      s = d * pow2(exponent(ke[tile])) * a.pre;
      if (a.cap > 0.0f) s = a.cap * tanh_of(s / a.cap);
      s -= slope * fabsf(static_cast<float>(pos - j));
    }
    float top = s;
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) {
      const float other = __shfl_xor(top, x, 64);
      top = top != top || other != other ? __uint_as_float(0x7fc00000u) : fmaxf(top, other);
    }
    const float next = top != top || m != m ? __uint_as_float(0x7fc00000u) : fmaxf(m, top);
    if (next == -INFINITY) continue;  // nothing seen yet
    const float f = m == next ? 1.0f : exp2f((m - next) * a.mul);
    const float p = see ? exp2f((s - next) * a.mul) : 0.0f;
    float sum = p;
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x, 64);
    l = l * f + sum;
    m = next;
#pragma unroll
    for (int c = 0; c < CPL; ++c) o[c] *= f;
    const uint64_t seen = __ballot(see);
    const float vs = pow2(exponent(ve[tile]));
    for (int x = 0; x < kKvBlock; ++x) {
      if (!((seen >> x) & 1)) continue;
      const float px = __shfl(p, x, 64) * vs;
      const uint8_t* vr = V + static_cast<size_t>(tile * kKvBlock + x) * D + CPL * lane;
#pragma unroll
      for (int c = 0; c < CPL; ++c) o[c] = fmaf(px, __builtin_amdgcn_cvt_f32_fp8(vr[c], 0), o[c]);
    }
  }
  const size_t pr = part_row(a, head, r, z);
#pragma unroll
  for (int c = 0; c < CPL; ++c) {
    const float v = l == 0.0f ? 0.0f : o[c] / l;
    if (a.splits == 1)
      a.out[row * D + CPL * lane + c] = static_cast<uint16_t>(f32_to_bf16_bits(v));
    else
      a.part[pr * D + CPL * lane + c] = v;
  }
  if (a.splits > 1 && lane == 0) a.ml[pr] = make_float2(m * a.mul, l);
}

// ---- scores and softmax, shared by the two matrix-core kernels
//
// S^T = K Q^T on the matrix cores: A = 16 keys, B = 16 rows, so that lane (n =
// lane % 16, g = lane / 16) ends with row n's scores of keys 16 b + 4 g + r of key
// block b.  Codes are converted to bf16 (exact); the keys' scale 2^ek multiplies the
// sums.  (The 8-bit matrix instructions would take the codes as they are, but align
// the products of a sum to 2^-14 or so of the largest.)
//   O^T += V^T P^T takes the probabilities where they are, contraction slot 4 h + r of
// lane group g being key 16 h + 4 g + r of 32, and codes converted to fp16 (exact).  A
// value block's 2^ev goes into the probability's exponent.  A probability enters as two
// fp16 parts, rounded and the rest rounded, 22 bits or more together: one would be off by
// up to 2^-11, more than all the fp32 steps before it.  The second part's products and
// sums cost nothing where the bytes bound the kernel and a tenth to a third of a prompt
// (2048 tokens 52.7 -> 63.6 us, 512 behind 32256 271 -> 351, packed documents 68 -> 75).
//
// A score's exponent is y = c S, c = mul 2^ek.  A row keeps its sum l = sum 2^(y - L) and O = sum
// 2^(y + ev - A) code; L and A are whole numbers, so that c S + ev - A is one fma
// that rounds once whatever their size, and rescaling by their changes is exact.  A
// makes the largest probability 2^6 to 2^7 when it is set: the smallest fp16 step, which
// ends the second part, is 2^-30 of the largest weighted value or less.  The sum is
// taken of the same parts by the matrix cores (a row of ones), in 32 bits.  Only if it
// overflows (a probability past fp16: 2^9 above the last maximum; the first keys of a
// row) is the maximum looked for, and L and A moved.  The sum knows no values: a block whose scale is so far below an earlier
// one's (zeros have the least) that n keys could lose it more than n 2^-28 of the
// largest weight is summed by itself, without 2^ev.  (L is at least the maximum that A
// was set by, so the weight 1 is 2^(kAim + ev - that block's ev) or more in the sum, and
// half the smallest fp16 step is 2^-25.)  Exponents past 2^24 (kHuge), where whole
// numbers are no longer exact, leave the row to attend_row.
constexpr float kAim = 7.0f;
constexpr int kFarBelow = 4;
constexpr float kNone = -3e38f;  // L and A of a row without keys
constexpr float kHuge = 16777216.0f;

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ msk::f32x4_t mfma_f16(f16x8_t a, f16x8_t b, msk::f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// maximum, NaN if one is
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// maximum over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float group_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = max_of(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_of(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The 16-byte pieces of a key row that a lane of group g holds, two contraction
// steps each.
constexpr int key_pieces(int D) { return D / 64; }
__device__ __forceinline__ int key_piece(int x, int g) { return 4 * x + g; }

__device__ __forceinline__ msk::bf16x8_t codes_bf16(uint32_t lo, uint32_t hi) {
  const uint2 a = codes_to_bf16(lo, 1.0f), b = codes_to_bf16(hi, 1.0f);
  return msk::as_bf16x8(make_uint4(a.x, a.y, b.x, b.y));
}

// A row of q as matrix operands, in the order of the pieces.
template <int D>
struct Query {
  msk::bf16x8_t part[2 * key_pieces(D)];
  __device__ __forceinline__ void load(const uint16_t* q, int g) {
#pragma unroll
    for (int x = 0; x < 2 * key_pieces(D); ++x)
      part[x] = msk::as_bf16x8(*reinterpret_cast<const uint4*>(q + 16 * key_piece(x / 2, g) + 8 * (x % 2)));
  }
};

template <int DB>
struct RowState {
  float l = 0.0f, L = kNone, A = kNone;
  msk::f32x4_t O[DB];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int c = 0; c < DB; ++c) O[c] = msk::f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // whether the row has to be left to attend_row
  __device__ __forceinline__ bool lost() const { return !isfinite(l) || (A != kNone && fabsf(A) > kHuge); }
};

// Probabilities of eight keys as matrix operands: rounded, and the rest rounded.
struct Prob {
  f16x8_t hi, lo;
};

// Two probabilities, those of the scores s0 and s1, in places 2 i and 2 i + 1.
__device__ __forceinline__ void softmax_pair(float s0, float s1, float c, float off, int i, Prob& p) {
  const f32x2_t e = {__builtin_amdgcn_exp2f(fmaf(s0, c, off)), __builtin_amdgcn_exp2f(fmaf(s1, c, off))};
  const f16x2_t hi = __builtin_convertvector(e, f16x2_t);
  p.hi[2 * i] = hi[0];
  p.hi[2 * i + 1] = hi[1];
  float minus = -1.0f;
  asm("" : "+s"(minus));  // unknown to the compiler, which makes one mixed fma of it and both conversions then
  p.lo[2 * i] = static_cast<_Float16>(fmaf(static_cast<float>(hi[0]), minus, e[0]));
  p.lo[2 * i + 1] = static_cast<_Float16>(fmaf(static_cast<float>(hi[1]), minus, e[1]));
}

// The probabilities of 2 H key blocks, H operands, and their sum for every row
// (all four values alike).
template <int H>
__device__ __forceinline__ msk::f32x4_t probabilities(const msk::f32x4_t (&S)[2 * H], float c, float off, Prob (&P)[H]) {
  const f16x8_t ones = {1, 1, 1, 1, 1, 1, 1, 1};
  msk::f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < H; ++h) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      softmax_pair(S[2 * h + i / 2][2 * (i % 2)], S[2 * h + i / 2][2 * (i % 2) + 1], c, off, i, P[h]);
    sum = mfma_f16(ones, P[h].hi, sum);
    sum = mfma_f16(ones, P[h].lo, sum);
  }
  return sum;
}

// The scale of the value blocks so far: whether one is far below an earlier one.
struct Far {
  int most = kExpMin;
  __device__ __forceinline__ bool below(int ev) {
    const bool far = ev < most - kFarBelow;
    most = max(most, ev);
    return far;
  }
};

// a row's largest exponent c S, -inf where it sees nothing
template <int NB>
__device__ __forceinline__ float top_of(const msk::f32x4_t (&S)[NB], float c) {
  float top = S[0][0];
#pragma unroll
  for (int k = 0; k < NB; ++k)
#pragma unroll
    for (int r = 0; r < 4; ++r) top = max_of(top, S[k][r]);
  return ceilf(group_max(top) * c);
}

// Softmax of QB rows' scores S of 2 H key blocks: their operands P, and what l, L, A
// and O become; far: their values are far below earlier ones (the same in every lane).
template <int QB, int DB, int H>
__device__ __forceinline__ void softmax_step(RowState<DB> (&st)[QB], const msk::f32x4_t (&S)[QB][2 * H], float c, float ev,
                                             bool far, Prob (&P)[QB][H]) {
  if (far) {
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      const float L = fmaxf(st[b].L, top_of(S[b], c));
      st[b].l = fmaf(probabilities<H>(S[b], c, kAim - L, P[b])[0], 0x1p-7f, st[b].l * __builtin_amdgcn_exp2f(st[b].L - L));
      st[b].L = L;
    }
  }
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    msk::f32x4_t sum = probabilities<H>(S[b], c, ev - st[b].A, P[b]);
    if (__any(!(sum[0] < INFINITY))) {
      const float top = top_of(S[b], c), L = fmaxf(st[b].L, top), A = fmaxf(st[b].A, top + ev - kAim);
      st[b].l *= __builtin_amdgcn_exp2f(st[b].L - L);
      const float f = __builtin_amdgcn_exp2f(st[b].A - A);
#pragma unroll
      for (int x = 0; x < DB; ++x) st[b].O[x] *= f;
      st[b].L = L;
      st[b].A = A;
      sum = probabilities<H>(S[b], c, ev - A, P[b]);
    }
    if (!far) st[b].l = fmaf(sum[0], __builtin_amdgcn_exp2f(st[b].A - ev - st[b].L), st[b].l);
  }
}

// A lane's row: what its scores and masks depend on.
struct Row {
  int pos, low, doc;  // position, the first that its window has
  float slope;
};
__device__ __forceinline__ Row row_of(const AttArgs& a, int head, const Span& sp, int r) {
  Row w;
  w.pos = sp.start + r / a.G;
  w.low = a.window > 0 ? max(w.pos - a.window + 1, 0) : 0;
  w.doc = a.docs ? a.docs[static_cast<size_t>(head / a.Hkv) * a.max_ctx + w.pos] : 0;
  w.slope = a.slopes ? a.slopes[head % a.Hkv * a.G + r % a.G] : 0.0f;
  return w;
}

// The documents of a lane's keys of NB key blocks.
template <int NB>
__device__ __forceinline__ void load_docs(const int32_t* docs, int k0, int4 (&d)[NB]) {
#pragma unroll
  for (int b = 0; b < NB; ++b) d[b] = *reinterpret_cast<const int4*>(docs + k0 + 16 * b + 4 * ((threadIdx.x & 63) >> 4));
}

// Raw scores of NB key blocks from key k0 on: scaled, capped and biased (a.scores)
// and masked (`masked`: some row of the wave may not see some of the keys; by_doc:
// by its document).
template <int NB>
__device__ __forceinline__ void modify(const AttArgs& a, const Row& w, int k0, int n, float ks, bool masked, bool by_doc,
                                       const int4 (&docs)[NB], msk::f32x4_t (&S)[NB]) {
  const int g4 = (threadIdx.x & 63) >> 4;
  if (a.scores) {
    float f = ks * a.pre;
    if (a.cap > 0.0f) {
      // Where all of a wave's scores are far below the cap, no exponential: 2048 tokens
      // behind 8192, 16 heads of 128 over 2, take 354 us, else 478 (261 without a cap).  Either
      // way a score has the same value, whatever the others of its wave, masked ones too.
      f *= 1.0f / a.cap;
      float top = 0.0f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          S[b][r] *= f;
          top = max_of(top, fabsf(S[b][r]));
        }
      if (__any(!(top < kSeries))) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[b][r] = a.cap * tanh_of(S[b][r]);
      } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[b][r] = a.cap * tanh_series(S[b][r]);
      }
      f = 1.0f;
    }
    if (a.slopes) {
      const float away = static_cast<float>(w.pos - k0 - 4 * g4);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[b][r] = fmaf(-w.slope, fabsf(away - static_cast<float>(16 * b + r)), S[b][r] * f);
    }
  }
  if (masked) {
    const int pre = min(a.prefix, n);
    const uint32_t span = static_cast<uint32_t>(w.pos - w.low);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = k0 + 16 * b + 4 * g4 + r;
        if (!(static_cast<uint32_t>(j - w.low) <= span || j < pre)) S[b][r] = -INFINITY;
      }
  }
  if (by_doc) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int d[4] = {docs[b].x, docs[b].y, docs[b].z, docs[b].w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (d[r] != w.doc || w.doc < 0) S[b][r] = -INFINITY;
    }
  }
}

__device__ __forceinline__ uint2 codes_to_f16(uint32_t c) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(c), 1.0f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(c), 1.0f, true)));
}
__device__ __forceinline__ uint4 codes_f16(uint32_t lo, uint32_t hi) {
  const uint2 a = codes_to_f16(lo), b = codes_to_f16(hi);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// Whether v holds in any thread of WAVES waves; flags: WAVES ints of LDS that no
// one else uses until the next barrier.
template <int WAVES>
__device__ __forceinline__ bool any_thread(bool v, int* flags) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool mine = __any(v);
  if (lane == 0) flags[wave] = mine;
  __syncthreads();
  int r = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) r |= flags[w];
  return r != 0;
}

// ---- few rows: one token, or a few
//
// At most 16 rows per key/value head (tokens x query heads of the group).  A
// work-group takes a head and a share of its tiles, a wave the steps (32 keys)
// w, w + NW, ... of the share, from a ring of its own (no barrier in the loop),
// and the waves' results are merged at the end.  Codes come to LDS by direct
// loads and become matrix operands when they are read: keys by 16-byte reads,
// values by transposing reads of eight keys of a column each.  16-byte piece p of
// row u sits in slot p ^ key_slot(u) or p ^ value_slot(u), so that the lanes
// which LDS serves together meet 16 different slots of 256 bytes.
//   Bound by the cache's bytes: 131000 keys of 8 heads of 128, 268 MB, take 42 us (6.4
// TB/s), 32 sequences of up to 8191 of 4 heads, 95 MB, 20.7; one token behind 1500 is
// bound by latency, 7 us.  Two stages a wave: at D = 64 they leave room for a second
// work-group per compute unit, 11.6 us for eight sequences' drafts of five against 16.4
// with three or four stages.
constexpr int kStep = 32;

template <int D>
__device__ __forceinline__ int key_slot(int u) { return (u / (256 / D)) & (D / 16 - 1); }
template <int D>
__device__ __forceinline__ int value_slot(int u) { return (((u & 7) | ((u >> 1) & 8)) / (256 / D)) & (D / 16 - 1); }

constexpr int few_waves(int D) { return D == 256 ? 4 : 8; }  // rings of eight at 256 are more than the LDS
constexpr int kFewStages = 2;

template <int D, bool MODS>
__global__ __launch_bounds__(64 * few_waves(D)) void attention_q_few_kernel(AttArgs a) {
  constexpr int NW = few_waves(D), NST = kFewStages, DB = D / 16;
  constexpr int PIECES = D / 16, RPL = 64 / PIECES;  // 16-byte pieces of a row, rows per load
  constexpr int KB = kStep * D, SB = 2 * KB, NK = KB / 1024, NL = 2 * NK;
  constexpr int PP = D + 4;                          // floats of a merged row
  static_assert((NST - 2) * NL < 64 && NW * NST * SB <= 160 * 1024, "rings");
  static_assert(NW * 16 * (PP + 3) * 4 + 64 <= NW * NST * SB, "the merge fits the rings");
  extern __shared__ __align__(16) unsigned char kv_lds[];
  const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.heads, z = blockIdx.x / a.heads, seq = head / a.Hkv;
  const Span sp = span_of(a.span, seq, a.pos0, a.T);
  if (sp.count == 0) return;
  const int rows = sp.count * a.G, n = sp.start + sp.count;
  const Tiles tl = tiles_of(a, sp.start, n - 1, n);
  const int total = tl.count();
  const int i0 = min(z * a.share, total), i1 = min(i0 + a.share, total);
  if (i0 == i1) {
    if (static_cast<int>(threadIdx.x) < rows) a.ml[part_row(a, head, threadIdx.x, z)] = make_float2(-INFINITY, 0.0f);
    return;
  }
  // the last tile's second half may be past the end
  const int steps = 2 * (i1 - i0) - (tl.at(i1 - 1) * kKvBlock + kStep >= n);
  const uint8_t *K = a.k + kv_row(a, head) * D, *V = a.v + kv_row(a, head) * D;
  const uint8_t *ke = a.k_exp + exp_row(a, head), *ve = a.v_exp + exp_row(a, head);
  const int32_t* docs = a.docs ? a.docs + static_cast<size_t>(seq) * a.max_ctx : nullptr;
  unsigned char* ring = kv_lds + wave * NST * SB;
  const uint32_t lbase = msk::lds_address(ring);
  const int lrow = lane / PIECES, slot = lane % PIECES;
  auto key0 = [&](int s) { return tl.at(i0 + (s >> 1)) * kKvBlock + (s & 1) * kStep; };
  auto issue = [&](int s, int buf) {  // steps past the wave's last reload the share's last one (never read)
    const int k0 = key0(min(s, steps - 1));
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      const int u = j * RPL + lrow;
      const size_t at = static_cast<size_t>(k0 + u) * D;
      msk::lds_load16(K + at + 16 * (slot ^ key_slot<D>(u)), lbase + buf * SB + 1024 * j);
      msk::lds_load16(V + at + 16 * (slot ^ value_slot<D>(u)), lbase + buf * SB + KB + 1024 * j);
    }
  };
  const int r = min(n16, rows - 1);
  const Row w = row_of(a, head, sp, r);
  Query<D> q[1];
  q[0].load(a.q + q_row(a, head, r) * D, g4);
#pragma unroll
  for (int p = 0; p < NST - 1; ++p) issue(wave + NW * p, p);
  Exps exps;
  Far far;
  int va;  // this lane's 8 bytes of column block 0
  {
    const int x = (lane >> 1) & 7, u = (x < 4 ? 0 : 12) + 4 * g4 + x;  // x >= 4: key 16 + 4 g + x - 4
    va = KB + u * D + 8 * (lane & 1);
  }
  const int vswz = value_slot<D>(((lane >> 1) & 7) < 4 ? 4 * g4 + ((lane >> 1) & 7) : 12 + 4 * g4 + ((lane >> 1) & 7));
  RowState<DB> st[1];
  st[0].clear();
  int cur = 0, nxt = NST - 1;
  for (int s = wave; s < steps; s += NW) {
    int ek, ve_s;
    exps.at(tl, i0, i1, i0 + (s >> 1), ke, ve, ek, ve_s);
    const int k0 = key0(s);
    int4 dj[2] = {};
    if (MODS && docs) load_docs(docs, k0, dj);
    msk::wait_vm<(NST - 2) * NL>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    issue(s + NW * (NST - 1), nxt);
    const unsigned char* sg = ring + cur * SB;
    cur = cur + 1 == NST ? 0 : cur + 1;
    nxt = nxt + 1 == NST ? 0 : nxt + 1;
    msk::f32x4_t S[1][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      S[0][b] = msk::f32x4_t{0.f, 0.f, 0.f, 0.f};
      const int u = 16 * b + n16;
      uint4 K[key_pieces(D)];
#pragma unroll
      for (int x = 0; x < key_pieces(D); ++x)
        K[x] = *reinterpret_cast<const uint4*>(sg + u * D + 16 * (key_piece(x, g4) ^ key_slot<D>(u)));
#pragma unroll
      for (int x = 0; x < key_pieces(D); ++x) {
        S[0][b] = msk::mfma16(codes_bf16(K[x].x, K[x].y), q[0].part[2 * x], S[0][b]);
        S[0][b] = msk::mfma16(codes_bf16(K[x].z, K[x].w), q[0].part[2 * x + 1], S[0][b]);
      }
    }
    const bool last = k0 + kStep > n;
    const float ks = pow2(ek), ev = static_cast<float>(ve_s);
    if constexpr (MODS) {
      modify(a, w, k0, n, ks, true, docs != nullptr, dj, S[0]);
    } else if (k0 + kStep > sp.start + 1) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (k0 + 16 * b + 4 * g4 + x > w.pos) S[0][b][x] = -INFINITY;
    }
    Prob P[1][1];
    softmax_step<1, DB, 1>(st, S, MODS && a.scores ? a.mul : a.mul * ks, ev, far.below(ve_s), P);
#pragma unroll
    for (int c = 0; c < DB; ++c) {
      uint2 t = msk::lds_read_tr8(sg + va + 16 * (c ^ vswz));
      if (last) {  // what lies past the end may be anything: code 0
        auto keep = [&](uint32_t x, int j) {
          const int m = n - j;
          return m >= 4 ? x : m <= 0 ? 0u : x & ((1u << (8 * m)) - 1);
        };
        t.x = keep(t.x, k0 + 4 * g4);
        t.y = keep(t.y, k0 + 16 + 4 * g4);
      }
      const uint2 lo = codes_to_f16(t.x), hi = codes_to_f16(t.y);
      const f16x8_t v = __builtin_bit_cast(f16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y));
      st[0].O[c] = mfma_f16(v, P[0][0].hi, st[0].O[c]);
      st[0].O[c] = mfma_f16(v, P[0][0].lo, st[0].O[c]);
    }
  }
  msk::wait_vm<0>();  // the reloads past the last step have landed
  __syncthreads();    // every wave is done with its ring
  float* part = reinterpret_cast<float*>(kv_lds);  // [NW][16][PP]
  float* mx = part + NW * 16 * PP;                 // [NW][16] L, then l and A
  float *sm = mx + NW * 16, *rx = sm + NW * 16;
  int* flags = reinterpret_cast<int*>(rx + NW * 16);
  bool bad = n16 < rows && st[0].lost();
  if (n16 < rows) {
    if (g4 == 0) {
      mx[wave * 16 + n16] = st[0].L;
      sm[wave * 16 + n16] = st[0].l;
      rx[wave * 16 + n16] = st[0].A;
    }
#pragma unroll
    for (int c = 0; c < DB; ++c)
      *reinterpret_cast<float4*>(part + (wave * 16 + n16) * PP + 16 * c + 4 * g4) =
          make_float4(st[0].O[c][0], st[0].O[c][1], st[0].O[c][2], st[0].O[c][3]);
  }
  __syncthreads();
  const int used = min(NW, steps);  // waves with a step
  constexpr int NV = 16 * D / (64 * NW);
  float val[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = k * 64 * NW + threadIdx.x, row = i / D, col = i % D;
    val[k] = 0.0f;
    if (row >= rows) continue;
    float top = mx[row];
    for (int x = 1; x < used; ++x) top = fmaxf(top, mx[x * 16 + row]);
    float num = 0.0f, den = 0.0f;
    for (int x = 0; x < used; ++x) {
      den += sm[x * 16 + row] * __builtin_amdgcn_exp2f(mx[x * 16 + row] - top);
      num += part[(x * 16 + row) * PP + col] * __builtin_amdgcn_exp2f(rx[x * 16 + row] - top);
    }
    val[k] = den == 0.0f ? 0.0f : num / den;
    bad |= !isfinite(val[k]);
    if (a.splits > 1 && col == 0) a.ml[part_row(a, head, row, z)] = make_float2(den == 0.0f ? -INFINITY : top, den);
  }
  if (any_thread<NW>(bad, flags)) {  // nothing of out is written yet: it may be q
    for (int row = wave; row < rows; row += NW) attend_row<D>(a, head, sp, row, tl, i0, i1, z, part + wave * D);
    return;
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = k * 64 * NW + threadIdx.x, row = i / D, col = i % D;
    if (row >= rows) continue;
    if (a.splits == 1)
      a.out[q_row(a, head, row) * D + col] = static_cast<uint16_t>(f32_to_bf16_bits(val[k]));
    else
      a.part[part_row(a, head, row, z) * D + col] = val[k];
  }
}

// ---- prompts
//
// A work-group takes 64 QB rows of one key/value head, a wave 16 QB of them, over
// its share of the tiles of 64 keys.  Codes come to LDS by direct loads, a tile
// ahead, and become operands when a wave reads them, as above: the conversions
// run beside the matrix instructions, and LDS holds and moves a byte per value.
//   Bound by the issue of vector and matrix instructions (311 and 104 a wave and tile of
// 32 rows): 512 tokens behind 32256, 32 heads over 8 of 128, take 351 to 363 us, 0.78
// PFLOP/s of products (1.2 with the probabilities' second parts); 2048 behind none 64, the
// 32 tiles of the longest block one after another.  Tiles converted once by all waves and
// kept in LDS as 16-bit values were slower, as were two groups of four waves with a share
// of the keys each (357 us for 338 of 2048 tokens behind 8192, probabilities in one part).
constexpr int kTileWaves = 4;
constexpr size_t tile_lds(int D) { return size_t{4} * kKvBlock * D; }  // two stages of keys and values

// Work-groups a compute unit: two by the registers of 128 rows, or of a width of 256.
template <int D, int QB, bool MODS>
__global__ __launch_bounds__(64 * kTileWaves, QB == 1 && D < 256 ? 3 : 2) void attention_q_tile_kernel(AttArgs a, int blocks) {
  constexpr int NW = kTileWaves, ROWS = 16 * NW * QB, DB = D / 16;
  constexpr int PIECES = D / 16, RPL = 64 / PIECES;  // 16-byte pieces of a row, rows per load
  constexpr int TILE = kKvBlock * D, NL = TILE / 1024 / NW;  // bytes of a tile's keys (or values), their loads per wave
  static_assert(NL >= 1 && NL * NW * 1024 == TILE, "loads");
  extern __shared__ __align__(16) unsigned char kv_lds[];
  __shared__ int doc_s[2 * NW], one_s[NW];
  __shared__ uint32_t near_s[NW], whole_s[NW];
  const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.heads, zj = blockIdx.x / a.heads, j = zj % blocks, z = zj / blocks, seq = head / a.Hkv;
  const Span sp = span_of(a.span, seq, a.pos0, a.T);
  const int rows = sp.count * a.G, n = sp.start + sp.count;
  const int r0 = (blocks - 1 - j) * ROWS;  // the longest row blocks first
  if (r0 >= rows) return;
  const int r1 = min(r0 + ROWS, rows);  // the work-group's rows
  const Tiles tl = tiles_of(a, sp.start + r0 / a.G, sp.start + (r1 - 1) / a.G, n);
  const int total = tl.count(), share = (total + a.splits - 1) / a.splits;
  const int i0 = min(z * share, total), i1 = min(i0 + share, total);
  if (i0 == i1) {
    if (r0 + static_cast<int>(threadIdx.x) < r1) a.ml[part_row(a, head, r0 + threadIdx.x, z)] = make_float2(-INFINITY, 0.0f);
    return;
  }
  const uint8_t *K = a.k + kv_row(a, head) * D, *V = a.v + kv_row(a, head) * D;
  const uint8_t *ke = a.k_exp + exp_row(a, head), *ve = a.v_exp + exp_row(a, head);
  const int32_t* docs = MODS && a.docs ? a.docs + static_cast<size_t>(seq) * a.max_ctx : nullptr;

  Row w[QB];
  Query<D> q[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int r = min(r0 + (wave * QB + b) * 16 + n16, r1 - 1);  // rows past the last repeat it (never stored)
    w[b] = row_of(a, head, sp, r);
    q[b].load(a.q + q_row(a, head, r) * D, g4);
  }

  // documents: only tiles with a key of a document between the rows' least and
  // largest are visited, and those whose keys are all of the rows' one document need
  // no look at it; 64 tiles are looked at at a time
  int d_min = INT32_MAX, d_max = -1, chunk = -1;
  uint64_t near = ~uint64_t{0}, whole = 0, was_whole = 0;  // was_whole: of the 64 before
  bool one = true;  // all rows are of one document
  if constexpr (MODS) {
    if (docs) {
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        one = one && w[b].doc >= 0;
        d_min = w[b].doc >= 0 ? min(d_min, w[b].doc) : d_min;
        d_max = max(d_max, w[b].doc);
      }
      one = __all(one);
#pragma unroll
      for (int x = 8; x >= 1; x >>= 1) {
        d_min = min(d_min, __shfl_xor(d_min, x, 64));
        d_max = max(d_max, __shfl_xor(d_max, x, 64));
      }
      if (lane == 0) {
        doc_s[wave] = d_min;
        doc_s[NW + wave] = d_max;
        one_s[wave] = one;
      }
      __syncthreads();
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        d_min = min(d_min, doc_s[x]);
        d_max = max(d_max, doc_s[NW + x]);
        one = one && one_s[x];
      }
      one = one && d_min == d_max;
    }
  }
  // the first tile to visit from i on (the same in every thread)
  auto advance = [&](int i) {
    if constexpr (MODS) {
      if (docs) {
        while (i < i1) {
          if ((i - i0) / 64 != chunk) {  // wave: 16 tiles, lane: a quarter of one
            chunk = (i - i0) / 64;
            const int t = i0 + 64 * chunk + 16 * wave + (lane >> 2);
            bool hit = false, all = true;
            if (t < i1) {
              const int4* d = reinterpret_cast<const int4*>(docs + tl.at(t) * kKvBlock + 16 * (lane & 3));
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int4 v = d[x];
                hit |= (v.x >= d_min && v.x <= d_max) || (v.y >= d_min && v.y <= d_max) || (v.z >= d_min && v.z <= d_max) ||
                       (v.w >= d_min && v.w <= d_max);
                all = all && v.x == d_min && v.y == d_min && v.z == d_min && v.w == d_min;
              }
            }
            uint64_t h = __ballot(hit), f = __ballot(all);
            h |= h >> 1;
            h |= h >> 2;  // bit 4 k: tile k
            f &= f >> 1;
            f &= f >> 2;
            uint32_t bits = 0, full = 0;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              bits |= static_cast<uint32_t>((h >> (4 * x)) & 1) << x;
              full |= static_cast<uint32_t>((f >> (4 * x)) & 1) << x;
            }
            __syncthreads();  // the chunk before is read
            if (lane == 0) {
              near_s[wave] = bits;
              whole_s[wave] = full;
            }
            __syncthreads();
            was_whole = whole;
            near = whole = 0;
#pragma unroll
            for (int x = 0; x < NW; ++x) {
              near |= static_cast<uint64_t>(near_s[x]) << (16 * x);
              whole |= static_cast<uint64_t>(whole_s[x]) << (16 * x);
            }
          }
          const uint64_t rest = near >> ((i - i0) & 63);
          if (rest) return i + static_cast<int>(__builtin_ctzll(rest));
          i = i0 + 64 * (chunk + 1);
        }
        return i1;
      }
    }
    return min(i, i1);
  };

  int at_k[NL], at_v[NL];  // this lane's bytes of its wave's loads
  uint32_t to[NL];
#pragma unroll
  for (int x = 0; x < NL; ++x) {
    const int u = (wave + NW * x) * RPL + lane / PIECES;
    at_k[x] = u * D + 16 * (lane % PIECES ^ key_slot<D>(u));
    at_v[x] = u * D + 16 * (lane % PIECES ^ value_slot<D>(u));
    to[x] = msk::lds_address(kv_lds) + (wave + NW * x) * 1024;
  }
  auto issue = [&](int i, int buf) {  // past the last tile: that one again (never read)
    const size_t k0 = static_cast<size_t>(tl.at(min(i, i1 - 1))) * kKvBlock * D;
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      msk::lds_load16(K + k0 + at_k[x], to[x] + buf * 2 * TILE);
      msk::lds_load16(V + k0 + at_v[x], to[x] + buf * 2 * TILE + TILE);
    }
  };
  // positions of the wave's first and last rows
  const int p_min = sp.start + min(r0 + wave * QB * 16, r1 - 1) / a.G;
  const int p_max = sp.start + min(r0 + (wave + 1) * QB * 16 - 1, r1 - 1) / a.G;
  constexpr int KP = key_pieces(D);
  const unsigned char* ka[KP];  // this lane's pieces of keys 0 .. 15
#pragma unroll
  for (int x = 0; x < KP; ++x) ka[x] = kv_lds + n16 * D + 16 * (key_piece(x, g4) ^ key_slot<D>(n16));
  const int vx = (lane >> 1) & 7, vrow = (vx < 4 ? 0 : 12) + 4 * g4 + vx;  // vx >= 4: key 16 + 4 g + vx - 4
  const unsigned char* const va = kv_lds + TILE + vrow * D + 8 * (lane & 1);
  const int vswz = value_slot<D>(vrow);
  RowState<DB> st[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) st[b].clear();

  int it = advance(i0), nx = advance(it + 1);  // this tile and the next
  Exps exps;
  Far far;
  auto step = [&](int p) {
    const int k0 = tl.at(it) * kKvBlock;
    int ek, ve_it;
    exps.at(tl, i0, i1, it, ke, ve, ek, ve_it);
    const float ks = pow2(ek), ev = static_cast<float>(ve_it);
    bool skip, masked;  // whether no row of the wave sees the tile, and whether some do not see all of it
    if constexpr (MODS) {
      skip = !((k0 <= p_max && (a.window <= 0 || k0 + kKvBlock - 1 > p_min - a.window)) || k0 < a.prefix);
      masked = !((k0 + kKvBlock - 1 <= p_min && (a.window <= 0 || p_max - k0 < a.window)) ||
                 (k0 + kKvBlock <= a.prefix && k0 + kKvBlock <= n));
    } else {
      skip = k0 > p_max;
      masked = k0 + kKvBlock - 1 > p_min;
    }
    int4 dj[4] = {};
    bool by_doc = false;
    if constexpr (MODS) {
      if (docs) {  // before the next tile's loads, which nothing waits for then
        const int d = it - i0;
        by_doc = !(one && (((d / 64 == chunk ? whole : was_whole) >> (d & 63)) & 1));
        if (by_doc && !skip) load_docs(docs, k0, dj);
      }
    }
    const int after = advance(nx + 1);
    msk::wait_vm<0>();
    msk::bare_barrier();  // the tile is staged, the other stage is read
    issue(nx, p ^ 1);
    if (n - k0 < kKvBlock) {  // values past the end may be anything: code 0
      for (int x = (n - k0) * D + 16 * threadIdx.x; x < TILE; x += 16 * 64 * NW)
        *reinterpret_cast<uint4*>(kv_lds + p * 2 * TILE + TILE + x) = make_uint4(0, 0, 0, 0);
      msk::bare_barrier();
    }
    if (!skip) {
      msk::f32x4_t S[QB][4];
      uint4 K4[4];
      auto key = [&](int f) { return *reinterpret_cast<const uint4*>(ka[f % KP] + p * 2 * TILE + f / KP * 16 * D); };
#pragma unroll
      for (int f = 0; f < 4; ++f) K4[f] = key(f);
#pragma unroll
      for (int f = 0; f < 4 * KP; ++f) {
        const uint4 k = K4[f % 4];
        const msk::bf16x8_t lo = codes_bf16(k.x, k.y), hi = codes_bf16(k.z, k.w);
        if (f + 4 < 4 * KP) K4[f % 4] = key(f + 4);
#pragma unroll
        for (int b = 0; b < QB; ++b)
          S[b][f / KP] = msk::mfma16(lo, q[b].part[f % KP * 2], f % KP == 0 ? msk::f32x4_t{0.f, 0.f, 0.f, 0.f} : S[b][f / KP]);
#pragma unroll
        for (int b = 0; b < QB; ++b) S[b][f / KP] = msk::mfma16(hi, q[b].part[f % KP * 2 + 1], S[b][f / KP]);
        __builtin_amdgcn_sched_barrier(0);  // no more operands at a time
      }
      auto value = [&](int f) {  // 16 columns of 32 keys
        return msk::lds_read_tr8(va + p * 2 * TILE + 32 * (f / DB) * D + 16 * ((f % DB) ^ vswz));
      };
      if constexpr (MODS) {
        if (masked || by_doc || a.scores) {
#pragma unroll
          for (int b = 0; b < QB; ++b) modify(a, w[b], k0, n, ks, masked, by_doc, dj, S[b]);
        }
      } else if (masked) {
#pragma unroll
        for (int b = 0; b < QB; ++b)
#pragma unroll
          for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (k0 + 16 * kb + 4 * g4 + x > w[b].pos) S[b][kb][x] = -INFINITY;
      }
      Prob P[QB][2];
      softmax_step<QB, DB, 2>(st, S, MODS && a.scores ? a.mul : a.mul * ks, ev, far.below(ve_it), P);
      uint2 V[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) V[f] = value(f);
      uint4 v = codes_f16(V[0].x, V[0].y);
#pragma unroll
      for (int f = 0; f < 2 * DB; ++f) {
        if (f + 4 < 2 * DB) V[f % 4] = value(f + 4);
        const uint2 next = V[(f + 1) % 4];
#pragma unroll
        for (int b = 0; b < QB; ++b) st[b].O[f % DB] = mfma_f16(__builtin_bit_cast(f16x8_t, v), P[b][f / DB].hi, st[b].O[f % DB]);
#pragma unroll
        for (int b = 0; b < QB; ++b) st[b].O[f % DB] = mfma_f16(__builtin_bit_cast(f16x8_t, v), P[b][f / DB].lo, st[b].O[f % DB]);
        if (f + 1 < 2 * DB) v = codes_f16(next.x, next.y);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    it = nx;
    nx = after;
  };
  if (it < i1) {
    issue(it, 0);
    for (;;) {
      step(0);
      if (it >= i1) break;
      step(1);
      if (it >= i1) break;
    }
    msk::wait_vm<0>();  // the reload past the last tile has landed
  }
  bool bad = false;
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const float f = st[b].l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(st[b].A - st[b].L) / st[b].l;
    bad |= st[b].lost();
#pragma unroll
    for (int c = 0; c < DB; ++c)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        st[b].O[c][x] *= f;
        bad |= !isfinite(st[b].O[c][x]);
      }
  }
  __syncthreads();  // LDS is free
  if (any_thread<NW>(bad, reinterpret_cast<int*>(kv_lds))) {  // nothing of out is written yet: it may be q
    __syncthreads();  // the flags are read
    for (int r = r0 + wave; r < r1; r += NW)
      attend_row<D>(a, head, sp, r, tl, i0, i1, z, reinterpret_cast<float*>(kv_lds) + wave * D);
    return;
  }
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const int r = r0 + (wave * QB + b) * 16 + n16;
    if (r >= r1) continue;
    if (a.splits == 1) {
      uint16_t* dst = a.out + q_row(a, head, r) * D + 4 * g4;
#pragma unroll
      for (int c = 0; c < DB; ++c)
        *reinterpret_cast<uint2*>(dst + 16 * c) =
            make_uint2(f32_to_bf16_bits(st[b].O[c][0]) | f32_to_bf16_bits(st[b].O[c][1]) << 16,
                       f32_to_bf16_bits(st[b].O[c][2]) | f32_to_bf16_bits(st[b].O[c][3]) << 16);
    } else {
      const size_t pr = part_row(a, head, r, z);
#pragma unroll
      for (int c = 0; c < DB; ++c)
        *reinterpret_cast<float4*>(a.part + pr * D + 16 * c + 4 * g4) =
            make_float4(st[b].O[c][0], st[b].O[c][1], st[b].O[c][2], st[b].O[c][3]);
      if (g4 == 0) a.ml[pr] = make_float2(st[b].l == 0.0f ? -INFINITY : st[b].L, st[b].l);
    }
  }
}

// ---- the splits of a row, joined
//
// WPR waves per row.  Every wave weighs the splits (lane = split); groups of D / 4
// lanes add up every NG-th of them.  Bound by latency for few rows (4.6 us for 32 rows of 64
// splits), by the results' bytes for many (10 us for 16384 rows of 4).  One wave a row and
// four, with the attention before them: 13.4 and 12.9 us with 128 rows, 282 and 295 with
// 16384.  Joined by the last work-group of a head instead, 131000 keys took 49.6 us for 46.2.
constexpr int kMostSplits = 64;
constexpr int kJoinThreads = 256;
constexpr int kJoinManyRows = 2048;

template <int D, int WPR>
__global__ __launch_bounds__(kJoinThreads) void attention_q_join_kernel(AttArgs a, int rows) {
  constexpr int COLS = D / 4, NG = 64 * WPR / COLS, RPW = kJoinThreads / 64 / WPR;  // rows of a work-group
  __shared__ __align__(16) float sums[RPW][NG][D];
  const int lane = threadIdx.x & 63, t = threadIdx.x % (64 * WPR), slot = threadIdx.x / (64 * WPR);
  const int row = blockIdx.x * RPW + slot, per = a.T * a.G, head = row / per, r = row % per;
  const bool in = row < rows && r < span_of(a.span, min(head, a.heads - 1) / a.Hkv, a.pos0, a.T).count * a.G;
  const size_t pr = part_row(a, head, r, 0);
  const float2 ml = in && lane < a.splits ? a.ml[pr + lane] : make_float2(-INFINITY, 0.0f);
  float top = ml.x;
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
  const float w = ml.x == top ? ml.y : ml.y * __builtin_amdgcn_exp2f(ml.x - top);
  float total = w;
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) total += __shfl_xor(total, x, 64);
  const int c = t % COLS, g = t / COLS;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int z0 = 0; z0 < a.splits; z0 += 4 * NG) {  // four loads in flight
    float f[4];
    float4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int z = z0 + i * NG + g;
      f[i] = __shfl(w, z & 63, 64);
      const float y = __shfl(ml.y, z & 63, 64);
      x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (in && z < a.splits && y != 0.0f)  // a share without keys: nothing was written
        x[i] = *reinterpret_cast<const float4*>(a.part + (pr + z) * D + 4 * c);
      else
        f[i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v.x = fmaf(f[i], x[i].x, v.x), v.y = fmaf(f[i], x[i].y, v.y), v.z = fmaf(f[i], x[i].z, v.z), v.w = fmaf(f[i], x[i].w, v.w);
  }
  if constexpr (NG > 1) {
    *reinterpret_cast<float4*>(&sums[slot][g][4 * c]) = v;
    __syncthreads();
    if (g == 0) {
#pragma unroll
      for (int x = 1; x < NG; ++x) {
        const float4 y = *reinterpret_cast<const float4*>(&sums[slot][x][4 * c]);
        v.x += y.x, v.y += y.y, v.z += y.z, v.w += y.w;
      }
    }
  }
  if (in && g == 0) {
    const float f = total == 0.0f ? 0.0f : 1.0f / total;
    *reinterpret_cast<uint2*>(a.out + q_row(a, head, r) * D + 4 * c) =
        make_uint2(f32_to_bf16_bits(v.x * f) | f32_to_bf16_bits(v.y * f) << 16,
                   f32_to_bf16_bits(v.z * f) | f32_to_bf16_bits(v.w * f) << 16);
  }
}

// How a call is run.
struct Plan {
  int variant;  // 0: attention_q_few_kernel, 1, 2: attention_q_tile_kernel of 64 or 128 rows
  int blocks;   // work-groups per head and split
  int splits;   // shares of a row's tiles
  int share;    // tiles of a share
};

// All that a call's splits depend on is rounded down, so that a window makes them no
// more than they are without it, and `spans` no fewer.
//   Few rows: a work-group per compute unit, two with spans (their sequences may be of
// any length), of at least two tiles: 32 sequences of 4000 keys, 32 heads over 8 of 128,
// take 42.9 us with 256 work-groups and 48.4 with 512; 8 sequences of up to 3001, drafts
// of five, 24 heads over 8 of 64, 17.1 and 14.6; one token behind 1500 10.0 us with
// shares of four tiles and 9.4 with two.  Below 2048 / D tiles they are not split, which
// saves the join: 32 heads over 8 of 128 at 700 keys 8.4 and 10.1 us, at 1000 9.6 and 9.8, at
// 1500 11.4 and 9.5; 16 over 4 of 256 at 400 14.0 and 13.8, at 700 17.3 and 14.2.
//   More: row blocks of 128 (more matrix instructions to a converted code) if their
// work-groups, with shares of sixteen tiles or more on average, fill the chip twice
// over, else of 64: 2048 tokens behind 8192, 32 heads over 8 of 128, 403 and 462 us; 512
// behind 4096 68.3 and 76.1; 4096 behind none 186 and 204; but 2048 behind none 64.0 and
// 59.2, 1024 32.6 and 23.5, and 100 10.1 and 7.5.
Plan plan_of(int64_t heads, int T, int G, int D, int pos0, bool spans, int window, int prefix) {
  Plan p;
  const int64_t rows = static_cast<int64_t>(T) * G;
  const int64_t all = (static_cast<int64_t>(pos0) + T + kKvBlock - 1) / kKvBlock;
  const int64_t mean = std::max<int64_t>(all - T / (2 * kKvBlock), 1);  // over the rows
  auto with = [&](int variant, int64_t block, int64_t target, int64_t least) {
    p.variant = variant;
    p.blocks = static_cast<int>((rows + block - 1) / block);
    int64_t most = all;  // tiles of a row block
    if (window > 0)
      most = std::min<int64_t>(all, (static_cast<int64_t>(window) + std::min<int64_t>(T, block / G + 2)) / kKvBlock + 3 +
                                        prefix / kKvBlock);
    p.splits = static_cast<int>(
        std::max<int64_t>(1, std::min<int64_t>({target / (heads * p.blocks), std::min(most, mean) / least, kMostSplits})));
    p.share = static_cast<int>((most + p.splits - 1) / p.splits);
    return heads * p.blocks * p.splits;
  };
  if (rows <= 16) {
    with(0, 16, spans ? 512 : 256, all * D < 2048 ? all : 2);
    return p;
  }
  const int64_t least = 4 + heads * rows / 2048;  // what a share costs to write and join
  if (D < 256 && with(2, 128, 512, std::max<int64_t>(least, 16)) >= 512) return p;
  with(1, 64, 512, least);
  return p;
}

template <int D>
ms_status launch_attention_q(const AttArgs& a, const Plan& p, bool mods, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.heads) * p.blocks * p.splits)), block(64 * kTileWaves);
  if (p.variant == 0) {
    constexpr size_t lds = static_cast<size_t>(few_waves(D)) * kFewStages * 2 * kStep * D;
    if (mods)
      hipLaunchKernelGGL((attention_q_few_kernel<D, true>), grid, dim3(64 * few_waves(D)), lds, s, a);
    else
      hipLaunchKernelGGL((attention_q_few_kernel<D, false>), grid, dim3(64 * few_waves(D)), lds, s, a);
  } else if (p.variant == 1) {
    if (mods)
      hipLaunchKernelGGL((attention_q_tile_kernel<D, 1, true>), grid, block, tile_lds(D), s, a, p.blocks);
    else
      hipLaunchKernelGGL((attention_q_tile_kernel<D, 1, false>), grid, block, tile_lds(D), s, a, p.blocks);
  } else if constexpr (D < 256) {
    if (mods)
      hipLaunchKernelGGL((attention_q_tile_kernel<D, 2, true>), grid, block, tile_lds(D), s, a, p.blocks);
    else
      hipLaunchKernelGGL((attention_q_tile_kernel<D, 2, false>), grid, block, tile_lds(D), s, a, p.blocks);
  }
  if (p.splits > 1) {
    const int rows = a.heads * a.T * a.G;
    if (rows >= kJoinManyRows)
      hipLaunchKernelGGL((attention_q_join_kernel<D, 1>), dim3((rows + 3) / 4), dim3(kJoinThreads), msk::kGuardLds, s, a, rows);
    else
      hipLaunchKernelGGL((attention_q_join_kernel<D, 4>), dim3(rows), dim3(kJoinThreads), msk::kGuardLds, s, a, rows);
  }
  return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP;
}

// rows of all sequences that a call may have: grids and row numbers stay in 31 bits
constexpr int64_t kMostRows = int64_t{1} << 22;

// [rows][splits] results of D floats, exponents and sums
uint64_t workspace_of(int64_t rows, int splits, int D) {
  return static_cast<uint64_t>(rows) * splits * (D + 2) * sizeof(float);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
ms_status launched() { return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP; }

ms_status check_cache(const ms_kv_cache_q* c) {
  if (!c || c->n_seqs <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->max_ctx <= 0) return MS_E_INVALID;
  if (c->max_ctx % kKvBlock != 0) return MS_E_INVALID;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return MS_E_UNSUPPORTED;
  return MS_OK;
}

bool cache_pointers(const ms_kv_cache_q* c) {
  return c->k && c->v && c->k_exp && c->v_exp && aligned16(c->k) && aligned16(c->v);
}

}  // namespace

extern "C" {

ms_status ms_rope_kv_q(const ms_kv_cache_q* cache, const ms_rope_desc* rope, const float* qkv, int32_t T, int32_t Hq,
                       int32_t pos0, const int32_t* span_dev, void* q_out, void* stream) {
  if (const ms_status st = check_cache(cache); st != MS_OK) return st;
  const int Hkv = cache->n_kv_heads, D = cache->head_dim;
  if (!rope || T < 0 || Hq <= 0 || Hq % Hkv != 0 || pos0 < 0) return MS_E_INVALID;
  if (!(rope->base > 1.0) || !std::isfinite(rope->base) || !(rope->factor >= 1.0) || !std::isfinite(rope->factor) ||
      !(rope->orig_ctx >= 0.0) || !std::isfinite(rope->orig_ctx) || !(rope->mscale > 0.0) ||
      !std::isfinite(static_cast<float>(rope->mscale)) ||
      rope->rot_dim < 0 || rope->rot_dim > D || rope->rot_dim % 2 != 0)
    return MS_E_INVALID;
  if (rope->orig_ctx > 0.0 && (!(rope->low >= 0.0) || !(rope->high > rope->low) || !std::isfinite(rope->high)))
    return MS_E_INVALID;
  if (static_cast<int64_t>(pos0) + T > cache->max_ctx) return MS_E_INVALID;
  if (T == 0) return MS_OK;
  if (!cache_pointers(cache) || !qkv || !q_out || !aligned16(qkv) || !aligned16(q_out)) return MS_E_INVALID;
  AppendArgs a;
  a.qkv = qkv;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k = static_cast<uint8_t*>(cache->k);
  a.v = static_cast<uint8_t*>(cache->v);
  a.k_exp = static_cast<uint8_t*>(cache->k_exp);
  a.v_exp = static_cast<uint8_t*>(cache->v_exp);
  a.span = span_dev;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.max_ctx = cache->max_ctx;
  a.pos0 = pos0;
  // blocks of 64 that T tokens touch: from pos0 on, or from anywhere
  a.blocks = span_dev ? (T + kKvBlock - 2) / kKvBlock + 1 : (pos0 + T - 1) / kKvBlock - pos0 / kKvBlock + 1;
  a.rot = rope->rot_dim;
  a.interleaved = rope->interleaved != 0;
  a.log2_base = std::log2(rope->base);
  a.inv_factor = 1.0 / rope->factor;
  a.turns = rope->orig_ctx / (2.0 * M_PI);
  a.low = rope->low;
  a.inv_ramp = rope->orig_ctx > 0.0 ? 1.0 / (rope->high - rope->low) : 0.0;
  a.mscale = rope->mscale;
  const int64_t heads = static_cast<int64_t>(Hq) + 2 * Hkv;
  if (heads > INT32_MAX) return MS_E_UNSUPPORTED;
  // heads that share a work-group's angles: as many as leave kAppendGroups work-groups, two
  // per compute unit.  2048 tokens of 48 heads: 28.1 us with 256, 22.0 with 512, 31.1 with
  // 1024; 16 pieces of 41 tokens 13.4, 9.7, 13.0.  (Heads of 128, all of them turned: LDS
  // admits two there, more where heads are narrower or turned in part.)
  const int64_t all = heads * a.blocks;  // at most 2^31 * 2^26; in steps, so that no product passes 64 bits
  const int threads = append_threads(D);
  if (all > UINT32_MAX / threads || all * cache->n_seqs > UINT32_MAX / threads) return MS_E_UNSUPPORTED;
  a.group = static_cast<int>(std::min<int64_t>(std::max<int64_t>(all * cache->n_seqs / kAppendGroups, 1), heads));
  const int64_t wgs = (heads + a.group - 1) / a.group * a.blocks * cache->n_seqs;
  const dim3 grid(static_cast<unsigned>(wgs)), block(threads);
  const size_t lds = 2 * sizeof(float2) * std::min(T, kKvBlock) * (a.rot / 2);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 64)
    hipLaunchKernelGGL(rope_kv_q_kernel<64>, grid, block, lds, s, a);
  else if (D == 128)
    hipLaunchKernelGGL(rope_kv_q_kernel<128>, grid, block, lds, s, a);
  else
    hipLaunchKernelGGL(rope_kv_q_kernel<256>, grid, block, lds, s, a);
  return launched();
}

ms_status ms_kv_read_q(const ms_kv_cache_q* cache, int32_t pos0, int32_t n, void* k_out, void* v_out, void* stream) {
  if (const ms_status st = check_cache(cache); st != MS_OK) return st;
  if (pos0 < 0 || n < 0 || static_cast<int64_t>(pos0) + n > cache->max_ctx) return MS_E_INVALID;
  if (n == 0) return MS_OK;
  if (!cache_pointers(cache) || !k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return MS_E_INVALID;
  const int64_t per_head = (static_cast<int64_t>(n) * (cache->head_dim / 16) + kReadThreads - 1) / kReadThreads;
  const int64_t rows = static_cast<int64_t>(cache->n_seqs) * cache->n_kv_heads;
  if (rows > INT32_MAX || rows * per_head > UINT32_MAX / kReadThreads) return MS_E_UNSUPPORTED;
  hipLaunchKernelGGL(kv_read_q_kernel, dim3(static_cast<unsigned>(rows * per_head)), dim3(kReadThreads), msk::kGuardLds,
                     static_cast<hipStream_t>(stream), static_cast<const uint8_t*>(cache->k),
                     static_cast<const uint8_t*>(cache->v), static_cast<const uint8_t*>(cache->k_exp),
                     static_cast<const uint8_t*>(cache->v_exp), cache->head_dim, cache->max_ctx, pos0, n,
                     static_cast<int>(per_head), static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out));
  return launched();
}

ms_status ms_attention_q_workspace(const ms_kv_cache_q* cache, int32_t T, int32_t Hq, int32_t pos0,
                                   uint64_t* bytes_out) {
  if (const ms_status st = check_cache(cache); st != MS_OK) return st;
  if (!bytes_out || T < 0 || Hq <= 0 || Hq % cache->n_kv_heads != 0 || pos0 < 0 ||
      static_cast<int64_t>(pos0) + T > cache->max_ctx)
    return MS_E_INVALID;
  *bytes_out = 0;
  if (T == 0) return MS_OK;
  const int64_t rows = static_cast<int64_t>(T) * Hq;
  if (rows > kMostRows || rows * cache->n_seqs > kMostRows) return MS_E_UNSUPPORTED;
  // without a window, which only makes the splits fewer, and with spans, which may make them more
  const Plan p = plan_of(static_cast<int64_t>(cache->n_seqs) * cache->n_kv_heads, T, Hq / cache->n_kv_heads, cache->head_dim,
                         pos0, true, 0, 0);
  if (p.splits > 1) *bytes_out = workspace_of(rows * cache->n_seqs, p.splits, cache->head_dim);
  return MS_OK;
}

ms_status ms_attention_q(const ms_kv_cache_q* cache, const void* q, int32_t T, int32_t Hq, int32_t pos0,
                         const int32_t* span_dev, const ms_attn_opts* opts, void* out, void* workspace_dev,
                         uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (const ms_status st = ms_attention_q_workspace(cache, T, Hq, pos0, &need); st != MS_OK) return st;
  if (opts && (!(opts->scale >= 0.0f) || !std::isfinite(opts->scale * kLog2e) || !(opts->softcap >= 0.0f) ||
               !std::isfinite(opts->softcap) || opts->window < 0 || opts->prefix < 0 || !aligned16(opts->docs_dev)))
    return MS_E_INVALID;
  if (T == 0) return MS_OK;
  if (!cache_pointers(cache) || !q || !out || !aligned16(q) || !aligned16(out)) return MS_E_INVALID;
  if (need > 0 && (!workspace_dev || !aligned16(workspace_dev) || workspace_bytes < need)) return MS_E_INVALID;
  const int D = cache->head_dim;
  const int64_t rows = static_cast<int64_t>(T) * Hq * cache->n_seqs;  // at most kMostRows
  const uint64_t bytes = static_cast<uint64_t>(rows) * D * sizeof(uint16_t);
  const auto qa = reinterpret_cast<uintptr_t>(q), oa = reinterpret_cast<uintptr_t>(out);
  if (qa != oa && qa < oa + bytes && oa < qa + bytes) return MS_E_INVALID;
  AttArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint8_t*>(cache->k);
  a.v = static_cast<const uint8_t*>(cache->v);
  a.k_exp = static_cast<const uint8_t*>(cache->k_exp);
  a.v_exp = static_cast<const uint8_t*>(cache->v_exp);
  a.span = span_dev;
  a.slopes = opts ? opts->slopes_dev : nullptr;
  a.docs = opts ? opts->docs_dev : nullptr;
  a.out = static_cast<uint16_t*>(out);
  a.T = T;
  a.Hq = Hq;
  a.Hkv = cache->n_kv_heads;
  a.G = Hq / cache->n_kv_heads;
  a.max_ctx = cache->max_ctx;
  a.pos0 = pos0;
  a.heads = cache->n_seqs * cache->n_kv_heads;
  a.window = opts ? opts->window : 0;
  a.prefix = opts ? opts->prefix : 0;
  a.cap = opts ? opts->softcap : 0.0f;
  const float scale = opts && opts->scale > 0.0f ? opts->scale : 1.0f / std::sqrt(static_cast<float>(D));
  const bool scores = a.cap > 0.0f || a.slopes;  // more than the product's scale
  a.scores = scores;
  a.pre = scores ? scale : 1.0f;
  a.mul = scores ? kLog2e : scale * kLog2e;
  const Plan p = plan_of(a.heads, T, a.G, D, pos0, span_dev != nullptr, a.window, a.prefix);
  if (p.splits > 1 && workspace_of(rows, p.splits, D) > need) return MS_E_INVALID;  // plan_of: never more
  a.splits = p.splits;
  a.share = p.share;
  a.part = static_cast<float*>(workspace_dev);
  a.ml = reinterpret_cast<float2*>(a.part + rows * p.splits * D);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool mods = scores || a.window > 0 || a.prefix > 0 || a.docs;
  if (D == 64) return launch_attention_q<64>(a, p, mods, s);
  if (D == 128) return launch_attention_q<128>(a, p, mods, s);
  return launch_attention_q<256>(a, p, mods, s);
}

}  // extern "C"
