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
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;  // NaN stays NaN
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
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
// positions, for one head (query heads alike, so that the grid is the same).
// Thread c of a row takes four consecutive values; keys and values stay in
// registers between the block's largest magnitude and their codes.  The angle
// p f is reduced to a fraction of a turn in double precision (a position of
// 2^20 and 24 bits after it fit); sine and cosine of the fraction are fp32.
constexpr int kAppendThreads = 256;

struct AppendArgs {
  const float* qkv;
  uint16_t* q_out;
  uint8_t *k, *v, *k_exp, *v_exp;
  const int32_t* span;
  int T, Hq, Hkv, max_ctx, pos0, blocks;
  int rot, interleaved;
  double log2_base, inv_factor, turns, low, inv_ramp;  // turns: orig_ctx / 2 pi, 0 for f / factor
  float mscale;
};

// turns per position of pair i
__device__ __forceinline__ double pair_turns(const AppendArgs& a, int i) {
  const double f = exp2(-2.0 * i / a.rot * a.log2_base);
  double keep = 0.0;
  if (a.turns > 0.0) keep = fmin(fmax((a.turns * f - a.low) * a.inv_ramp, 0.0), 1.0);
  return f * ((1.0 - keep) * a.inv_factor + keep) * 0.15915494309189535;
}

template <int D>
__global__ __launch_bounds__(kAppendThreads) void rope_kv_q_kernel(AppendArgs a) {
  constexpr int COLS = D / 4, ROWS = kAppendThreads / COLS, PASSES = kKvBlock / ROWS;
  __shared__ uint32_t top_s[kAppendThreads / 64];
  const int heads = a.Hq + 2 * a.Hkv;
  const int b = blockIdx.x % a.blocks, head = blockIdx.x / a.blocks % heads, seq = blockIdx.x / a.blocks / heads;
  const Span sp = span_of(a.span, seq, a.pos0, a.T);
  const int base = (sp.start / kKvBlock + b) * kKvBlock;
  const int lo = max(sp.start, base), hi = min(sp.start + sp.count, base + kKvBlock);
  if (lo >= hi) return;  // uniform
  const int c4 = threadIdx.x % COLS, r0 = threadIdx.x / COLS, j0 = 4 * c4, half = a.rot / 2;
  const float* src = a.qkv + (static_cast<size_t>(seq) * a.T * heads + head) * D + j0;
  const size_t pitch = static_cast<size_t>(heads) * D;
  const bool turn = head < a.Hq + a.Hkv && j0 < a.rot;
  double f[4];
  if (turn) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = min(j0 + e, a.rot - 1);
      f[e] = pair_turns(a, a.interleaved ? j / 2 : j < half ? j : j - half);
    }
  }
  float val[PASSES][4];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int p = base + i * ROWS + r0;
    const bool in = p >= lo && p < hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) val[i][e] = 0.0f;
    if (!in) continue;
    const float* x = src + (p - sp.start) * pitch;
    const float4 own = *reinterpret_cast<const float4*>(x);
    val[i][0] = own.x, val[i][1] = own.y, val[i][2] = own.z, val[i][3] = own.w;
    if (turn) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + e;
        y[e] = val[i][e];
        if (j >= a.rot) continue;
        double t = p * f[e];
        t -= rint(t);
        float s, c;
        sincospif(2.0f * static_cast<float>(t), &s, &c);
        c *= a.mscale;
        s *= a.mscale;
        const bool first = a.interleaved ? !(j & 1) : j < half;
        const float other = a.interleaved ? val[i][e ^ 1] : x[first ? e + half : e - half];
        y[e] = val[i][e] * c + (first ? -other * s : other * s);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) val[i][e] = y[e];
    }
    if (head < a.Hq) {
      *reinterpret_cast<uint2*>(a.q_out + ((static_cast<size_t>(seq) * a.T + (p - sp.start)) * a.Hq + head) * D + j0) =
          make_uint2(f32_to_bf16_bits(val[i][0]) | f32_to_bf16_bits(val[i][1]) << 16,
                     f32_to_bf16_bits(val[i][2]) | f32_to_bf16_bits(val[i][3]) << 16);
    }
  }
  if (head < a.Hq) return;  // uniform
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
  const bool value = head >= a.Hq + a.Hkv;
  const size_t row = static_cast<size_t>(seq) * a.Hkv + (value ? head - a.Hq - a.Hkv : head - a.Hq);
  uint8_t* exps = (value ? a.v_exp : a.k_exp) + row * (a.max_ctx / kKvBlock) + base / kKvBlock;
  uint8_t* out = (value ? a.v : a.k) + (row * a.max_ctx + base) * D;
  const int was = lo > base ? exponent(*exps) : kExpMin;
  if ((threadIdx.x & 63) == 0) top_s[threadIdx.x >> 6] = top;
  __syncthreads();  // every thread has read the old exponent too
#pragma unroll
  for (int w = 0; w < kAppendThreads / 64; ++w) top = max(top, top_s[w]);
  // top = m 2^x, 1 <= m < 2, and 448 = 1.75 * 2^8; zero and subnormal magnitudes end at kExpMin
  int ex = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
  ex = max(min(max(ex, kExpMin), kExpMax), was);
  if (threadIdx.x == 0) *exps = static_cast<uint8_t>(ex + kExpBias);
  const float scale = pow2(-ex);
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int p = base + i * ROWS + r0;
    if (p >= lo && p < hi) *reinterpret_cast<uint32_t*>(out + static_cast<size_t>(p - base) * D + j0) = encode4(val[i], scale);
  }
  if (lo > base && ex > was) {  // the positions before the append, at the new exponent
    const float down = pow2(was - ex);
    for (int i = threadIdx.x; i < (lo - base) * COLS; i += kAppendThreads) {
      uint32_t* w = reinterpret_cast<uint32_t*>(out) + i;
      float v[4];
      decode4(*w, v);
      *w = encode4(v, down);
    }
  }
}

// ------------------------------------------------------------- read back
//
// 16 codes per thread.
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
  int T, Hq, Hkv, G, max_ctx, pos0;
  int window, prefix;
  float scale, cap;
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

// tanh, relative error below 2^-20: its series near zero, where the
// difference of exponentials would cancel
__device__ __forceinline__ float tanh_of(float x) {
  const float y = x * x;
  const float series = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  const float e = __builtin_amdgcn_exp2f(fabsf(x) * (-2.0f * kLog2e));
  const float far = (1.0f - e) / (1.0f + e);
  return fabsf(x) < 0.25f ? series : copysignf(far, x);
}

// Whether the query at position i (document di) sees key j of n (document dj).
__device__ __forceinline__ bool sees(const AttArgs& a, int i, int j, int n, int di, int dj) {
  const int d = i - j;
  bool s = (d >= 0 && (a.window <= 0 || d < a.window)) || j < a.prefix;
  s = s && j < n;
  if (a.docs) s = s && di == dj && di >= 0;
  return s;
}

// One query row by one wave: lane j of a tile has key j's score, then D / 64
// columns of the output.  Every value is read for the rows that see it only.
template <int D>
__device__ __forceinline__ void attend_row(const AttArgs& a, int seq, const Span& sp, int g, int t, int h, float* qs) {
  constexpr int CPL = D / 64;
  const int lane = threadIdx.x & 63;
  const int pos = sp.start + t, n = sp.start + sp.count, head = g * a.G + h;
  const size_t row = (static_cast<size_t>(seq) * a.T + t) * a.Hq + head;
#pragma unroll
  for (int c = 0; c < CPL; ++c) qs[CPL * lane + c] = __uint_as_float(static_cast<uint32_t>(a.q[row * D + CPL * lane + c]) << 16);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own row
  const size_t kv = static_cast<size_t>(seq) * a.Hkv + g;
  const uint8_t *K = a.k + kv * a.max_ctx * D, *V = a.v + kv * a.max_ctx * D;
  const uint8_t *ke = a.k_exp + kv * (a.max_ctx / kKvBlock), *ve = a.v_exp + kv * (a.max_ctx / kKvBlock);
  const int32_t* docs = a.docs ? a.docs + static_cast<size_t>(seq) * a.max_ctx : nullptr;
  const int di = docs ? docs[pos] : 0;
  const float slope = a.slopes ? a.slopes[head] : 0.0f;
  const Tiles tl = tiles_of(a, pos, pos, n);
  float m = -INFINITY, l = 0.0f, o[CPL] = {};
  for (int i = 0; i < tl.count(); ++i) {
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
      s = d * pow2(exponent(ke[tile])) * a.scale;
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
    const float f = m == next ? 1.0f : expf(m - next);
    const float p = see ? expf(s - next) : 0.0f;
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
#pragma unroll
  for (int c = 0; c < CPL; ++c)
    a.out[row * D + CPL * lane + c] = static_cast<uint16_t>(f32_to_bf16_bits(l == 0.0f ? 0.0f : o[c] / l));
}

constexpr int kRowThreads = 256;
template <int D>
__global__ __launch_bounds__(kRowThreads) void attention_q_kernel(AttArgs a, int seqs) {
  __shared__ float qs[kRowThreads / 64][D];
  const int wave = threadIdx.x >> 6;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 64) + wave;
  const int t = static_cast<int>(row / a.Hq % a.T), head = static_cast<int>(row % a.Hq);
  const int64_t seq = row / a.Hq / a.T;
  if (seq >= seqs) return;
  const Span sp = span_of(a.span, static_cast<int>(seq), a.pos0, a.T);
  if (t >= sp.count) return;
  attend_row<D>(a, static_cast<int>(seq), sp, head / a.G, t, head % a.G, qs[wave]);
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
      !(rope->orig_ctx >= 0.0) || !std::isfinite(rope->orig_ctx) || !(rope->mscale > 0.0) || !std::isfinite(rope->mscale) ||
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
  a.mscale = static_cast<float>(rope->mscale);
  const int64_t heads = static_cast<int64_t>(Hq) + 2 * Hkv;
  // in steps, so that no product passes 64 bits
  const int64_t wgs = heads * a.blocks;
  if (heads > INT32_MAX || wgs > UINT32_MAX / kAppendThreads || wgs * cache->n_seqs > UINT32_MAX / kAppendThreads)
    return MS_E_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(wgs * cache->n_seqs)), block(kAppendThreads);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 64)
    hipLaunchKernelGGL(rope_kv_q_kernel<64>, grid, block, 0, s, a);
  else if (D == 128)
    hipLaunchKernelGGL(rope_kv_q_kernel<128>, grid, block, 0, s, a);
  else
    hipLaunchKernelGGL(rope_kv_q_kernel<256>, grid, block, 0, s, a);
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
  return MS_OK;
}

ms_status ms_attention_q(const ms_kv_cache_q* cache, const void* q, int32_t T, int32_t Hq, int32_t pos0,
                         const int32_t* span_dev, const ms_attn_opts* opts, void* out, void* workspace_dev,
                         uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (const ms_status st = ms_attention_q_workspace(cache, T, Hq, pos0, &need); st != MS_OK) return st;
  if (opts && (!(opts->scale >= 0.0f) || !std::isfinite(opts->scale) || !(opts->softcap >= 0.0f) ||
               !std::isfinite(opts->softcap) || opts->window < 0 || opts->prefix < 0))
    return MS_E_INVALID;
  if (T == 0) return MS_OK;
  if (!cache_pointers(cache) || !q || !out || !aligned16(q) || !aligned16(out)) return MS_E_INVALID;
  if (need > 0 && (!workspace_dev || !aligned16(workspace_dev) || workspace_bytes < need)) return MS_E_INVALID;
  const int D = cache->head_dim;
  const int64_t rows = static_cast<int64_t>(T) * Hq;  // of a sequence
  constexpr int64_t kMostRows = int64_t{1} << 31;
  if (rows > kMostRows || rows * cache->n_seqs > kMostRows) return MS_E_UNSUPPORTED;
  const uint64_t bytes = static_cast<uint64_t>(rows) * cache->n_seqs * D * sizeof(uint16_t);
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
  a.window = opts ? opts->window : 0;
  a.prefix = opts ? opts->prefix : 0;
  a.scale = opts && opts->scale > 0.0f ? opts->scale : 1.0f / std::sqrt(static_cast<float>(D));
  a.cap = opts ? opts->softcap : 0.0f;
  constexpr int kWaves = kRowThreads / 64;
  const int64_t wgs = (rows * cache->n_seqs + kWaves - 1) / kWaves;
  if (wgs > UINT32_MAX / kRowThreads) return MS_E_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(wgs)), block(kRowThreads);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (D == 64)
    hipLaunchKernelGGL(attention_q_kernel<64>, grid, block, 0, s, a, cache->n_seqs);
  else if (D == 128)
    hipLaunchKernelGGL(attention_q_kernel<128>, grid, block, 0, s, a, cache->n_seqs);
  else
    hipLaunchKernelGGL(attention_q_kernel<256>, grid, block, 0, s, a, cache->n_seqs);
  return launched();
}

}  // extern "C"
