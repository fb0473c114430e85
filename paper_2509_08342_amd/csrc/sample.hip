// A token drawn from each row of logits: temperature, top-k, top-p and min-p, from given
// random numbers.  Stateless, like the other calls of the decoder loop.
//
// With the logits l in descending order, ties to the lower index, and weights
// exp((l - max) / temperature), every filter keeps a prefix, so the kept mass M is the least
// of the filters' masses, and the token is the first whose running mass passes u M: top-k
// keeps the mass of the first k, top-p of the fewest that reach p of that, min-p of the weights
// from min-p on.  No row is sorted: a histogram over the distance from the maximum gives the
// running mass at 4096 borders; only the tokens of the few bins in which a filter or the drawn
// mass ends are gathered and sorted.
//
// Weights are whole numbers of 2^-45, computed in double precision: their sums do not depend
// on the order of additions (so atomics may build them), and a border between two tokens is
// off by 2^-46 of the largest weight per token before it, where fp32 sums of 10^5 tokens
// would move it by more than the smallest tokens' weights.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <iterator>
#include <type_traits>

#include "kernels.h"
#include "moesplit.h"

namespace {

using msk::overlap;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;  // as many as a row of lanes
// (8192 bins sort fewer tokens and take longer to scan and merge: 64 rows of 131071 logits 44-50 us
// rather than 40-43.)
constexpr int kBins = 4096;
constexpr int kList = kThreads;  // gathered tokens
constexpr int kSubBins = 1024;   // of rows whose tokens crowd into few bins
constexpr int kMostTokens = (1 << 19) - 1;  // n 2^45 < 2^64
constexpr double kUnit = 35184372088832.0;  // 2^45
constexpr int kCus = 256, kXcds = 8;
constexpr double kFar = 46 * 256;  // 2^-46 rounds to zero units (in 256ths of powers of two)

// A logit as it counts: NaN where it is infinite (no comparison with NaN holds, and its weight is 0);
// where the largest is infinite, its likes are 0 and all others NaN.
__device__ __forceinline__ float logit(float x, bool infinite) {
  return infinite ? (x == INFINITY ? 0.0f : NAN) : fmaf(x, 0.0f, x);
}

// order of fp32 values as unsigned numbers; -0 and 0 alike
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Sums and scans of a wave by DPP moves, a tenth of a shuffle's latency.  moved(x): a lane's value
// goes on as CTRL says, to the rows of 16 lanes in ROWS; other lanes get 0.
enum { kShr = 0x110, kRor = 0x120, kNextRow = 0x142, kNextRows = 0x143 };
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t moved(uint32_t x, uint32_t other = 0) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(other), static_cast<int>(x), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t moved(uint64_t x) {
  return static_cast<uint64_t>(moved<CTRL, ROWS>(static_cast<uint32_t>(x >> 32))) << 32 | moved<CTRL, ROWS>(static_cast<uint32_t>(x));
}
// of the lanes up to each
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
  x += moved<kShr + 1>(x);
  x += moved<kShr + 2>(x);
  x += moved<kShr + 4>(x);
  x += moved<kShr + 8>(x);
  x += moved<kNextRow, 0xa>(x);
  return x + moved<kNextRows, 0xc>(x);
}
// of 16 lanes, to each
template <typename T>
__device__ __forceinline__ T row_sum(T x) {
  x += moved<kRor + 8>(x);
  x += moved<kRor + 4>(x);
  x += moved<kRor + 2>(x);
  return x + moved<kRor + 1>(x);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float moved(float x) {  // or stays
  return __uint_as_float(moved<CTRL, ROWS>(__float_as_uint(x), __float_as_uint(x)));
}
template <typename F>
__device__ __forceinline__ float wave_reduce(float x, F f) {
  x = f(x, moved<kRor + 8>(x));
  x = f(x, moved<kRor + 4>(x));
  x = f(x, moved<kRor + 2>(x));
  x = f(x, moved<kRor + 1>(x));
  x = f(x, moved<kNextRow, 0xa>(x));
  x = f(x, moved<kNextRows, 0xc>(x));
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
}
// A value that the lanes of a wave share, kept in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(uniform(__float_as_uint(x))); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return static_cast<uint64_t>(uniform(static_cast<uint32_t>(x >> 32))) << 32 | uniform(static_cast<uint32_t>(x));
}
__device__ __forceinline__ double uniform(double x) { return __longlong_as_double(uniform(static_cast<uint64_t>(__double_as_longlong(x)))); }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }

// of groups of P lanes (a power of two, the same in the wave), to each
template <typename T>
__device__ __forceinline__ T group_sum(T x, int P) {
  enum { kPairs = 0xb1, kFours = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140 };
  if (P > 1) x += moved<kPairs>(x);
  if (P > 2) x += moved<kFours>(x);
  if (P > 4) x += moved<kMirror8>(x);
  if (P > 8) x += moved<kMirror16>(x);
  if (P > 16) x += __shfl_xor(x, 16, 64);
  if (P > 32) x += __shfl_xor(x, 32, 64);
  return x;
}

// What a row's tokens are weighed with.
constexpr int kPowers = 256;
constexpr double kLn2 = 0.69314718055994530942;
struct Scale {
  double inv;   // kPowers / (ln 2 temperature)
  double top;   // the largest logit (finite)
  float half;   // half of it
  float bins;   // per half a unit of logits
  const double* powers;  // 2^(45 + i / kPowers)

  // by the distance from the maximum in fp32: never less for a smaller logit (of halves, as a
  // difference may pass the largest number)
  __device__ __forceinline__ float distance(float l) const { return fmaf(-0.5f, l, half) * bins; }
  __device__ __forceinline__ int bin(float l) const { return static_cast<int>(fminf(distance(l), kBins - 1)); }
  // exp((l - top) / temperature) in units: 2^(j / kPowers) from the table and the series of the
  // rest, |r| <= 1/2, to its fourth power (the next term is 2^-54)
  __device__ __forceinline__ uint64_t weight(float l) const {
    const double y = fmax((l - top) * inv, -kFar - kPowers);  // (NaN, of an endless temperature, too)
    constexpr double L = kLn2 / kPowers;
    constexpr double kWhole = 6755399441055744.0;  // 1.5 2^52: a sum with it is rounded to whole numbers
    const double z = y + kWhole, r = y - (z - kWhole);
    double s = fma(r, L * L * L * L / 24, L * L * L / 6);
    s = fma(r, s, L * L / 2);
    s = fma(r, s, L);
    s = fma(r, s, 1.0);
    const int i = __double2loint(z);
    const double e = s * powers[i & (kPowers - 1)];
    const double scaled = __hiloint2double(__double2hiint(e) + ((i & -kPowers) << 12), __double2loint(e));  // times 2^(i / kPowers), rounded down
    // rounds to a whole number in the low bits
    return static_cast<uint64_t>(__double_as_longlong(scaled + 4503599627370496.0)) & ((1ull << 52) - 1);
  }
};

struct SampleArgs {
  const float *logits, *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* idx;
  float* prob;
  int T, n;
  int splits, share;  // work-groups of a row, and their logits
  void* workspace;
};

// A gathered token: its order (a larger one comes earlier) and weight.
struct Token {
  uint64_t order;  // order_key, then bin and the index's complement: 13 and 19 bits
  uint64_t weight;
};

struct RangeShared {
  float wave_top[kWaves], wave_low[kWaves];
};
struct Shared : RangeShared {
  uint64_t mass[kBins];   // then exclusive sums
  uint32_t count[kBins];
  union {
    struct {  // gathered tokens, and their places in descending order
      uint64_t order[kList], weight[kList];
      uint32_t sorted[kList];
    };
    struct {
      uint64_t mass[kSubBins];
      uint32_t count[kSubBins];
    } sub;
  };
  float near[kList];       // tokens before they are weighed: the logit and the index
  int32_t near_at[kList];
  double powers[kPowers];
  uint64_t wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  uint64_t all, least;
  struct {
    uint64_t mass, weight;
    int32_t at;
  } found[3];
  uint32_t all_count, n_list, n_near, key_low, key_top;
  int32_t at;  // of the arg max
  int32_t found_bin[3][2];
};

// Exclusive sums of mass and count in place; the totals to sh.all and sh.all_count.  Returns
// the sums before and behind the thread's own bins, which follow each other.
struct Span {
  uint64_t mass0, mass1;
  uint32_t count0, count1;
};
template <int BINS, bool MASS, bool COUNT>
__device__ __forceinline__ Span scan_bins(Shared& sh, uint64_t* mass, uint32_t* count, uint64_t mass0, uint32_t count0) {
  constexpr int PER = BINS / kThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t x[PER], m = 0;
  uint32_t y[PER], c = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (MASS) m += x[i] = mass[tid * PER + i];
    if (COUNT) c += y[i] = count[tid * PER + i];
  }
  const uint64_t im = MASS ? wave_scan(m) : 0;
  const uint32_t ic = COUNT ? wave_scan(c) : 0;
  if (lane == 63) sh.wave_mass[wave] = im, sh.wave_count[wave] = ic;
  __syncthreads();
  const bool earlier = lane % kWaves < wave;
  uint64_t base = mass0 + (MASS ? row_sum(earlier ? sh.wave_mass[lane % kWaves] : 0) : 0) + im - m;
  uint32_t bc = count0 + (COUNT ? row_sum(earlier ? sh.wave_count[lane % kWaves] : 0) : 0) + ic - c;
  const Span own = {base, base + m, bc, bc + c};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (MASS) mass[tid * PER + i] = base, base += x[i];
    if (COUNT) count[tid * PER + i] = bc, bc += y[i];
  }
  if (tid == kThreads - 1) {
    if (MASS) sh.all = base;
    if (COUNT) sh.all_count = bc;
  }
  __syncthreads();
  return own;
}

// Where a prefix ends: at the token that makes it t long, that takes its mass to t, or past t.  As
// whole numbers: the prefix before is short of `length`, or of `mass`.
enum Cut { kCount, kReach, kPass };
struct Limit {
  Cut cut;
  uint64_t mass;
  uint32_t length;

  __device__ __forceinline__ bool is_short(uint64_t m, uint32_t n) const { return cut == kCount ? n < length : m < mass; }
};
__device__ __forceinline__ Limit limit(Cut cut, double t) {  // 0 <= t < 2^64
  const uint64_t m = uniform(static_cast<uint64_t>(cut == kPass ? floor(t) : ceil(t)));
  return {cut, m + (cut == kPass), static_cast<uint32_t>(min(m, static_cast<uint64_t>(UINT32_MAX)))};
}

// The bins in which the cuts at l0 and l1 lie, from exclusive sums: of the threads whose bins
// they may be in exactly one looks (the last where rounding leaves none).
template <int BINS>  // (found_bin[cut] has to be free)
__device__ __forceinline__ int2 bins_of(Shared& sh, const uint64_t* mass, const uint32_t* count, const Span& own, const Limit& l0, const Limit& l1) {
  constexpr int PER = BINS / kThreads;
  const int tid = threadIdx.x;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Limit& l = i ? l1 : l0;
    if ((tid == 0 || l.is_short(own.mass0, own.count0)) && (tid == kThreads - 1 || !l.is_short(own.mass1, own.count1))) {
      int b = tid * PER;
#pragma unroll
      for (int j = 1; j < PER; ++j)
        if (l.is_short(mass[tid * PER + j], count[tid * PER + j])) b = tid * PER + j;
      sh.found_bin[l.cut][i] = b;
    }
  }
  __syncthreads();
  return make_int2(sh.found_bin[l0.cut][0], sh.found_bin[l0.cut][1]);
}

struct End {
  uint64_t mass, weight;  // of the prefix, the token at its end included, and of that token
  int token;
};

// A thread's logits of [i0, i1) of a row: held in registers for all passes, or read again for each,
// AT_ONCE at a time.
constexpr int kHold = 32, kRead = 8;
template <int AT_ONCE>
struct Logits {
  static constexpr bool HELD = AT_ONCE == kHold;  // i1 - i0 <= kHold * kThreads
  const float* row;
  int i0, i1;
  bool infinite;
  float x[AT_ONCE];

  __device__ __forceinline__ void fetch(int from) {  // from + thread, from + thread + kThreads, ...
    steps<8>(from, [&](int g) {
#pragma unroll
      for (int i = g; i < g + 8; ++i) {
        const uint32_t at = 4u * min(from + i * kThreads + static_cast<int>(threadIdx.x), i1 - 1);  // (less than 2^21)
        x[i] = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(row) + at);
      }
    });
  }
  __device__ __forceinline__ void end(int from) {  // NaN past the end
#pragma unroll
    for (int g = 0; g < AT_ONCE; g += 8) {
      if (from + (g + 8) * kThreads <= i1) continue;
#pragma unroll
      for (int i = g; i < g + 8; ++i)
        if (from + i * kThreads + static_cast<int>(threadIdx.x) >= i1) x[i] = NAN;
    }
  }
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) x[i] = logit(x[i], infinite);
  }
  __device__ __forceinline__ Logits(const float* r, int from, int to) : row(r), i0(from), i1(to), infinite(false) {
    if (HELD) fetch(i0);
  }
  // Before the first pass: the largest, and the smallest that is finite.
  __device__ __forceinline__ float2 range() {
    float top = -INFINITY, low = INFINITY;
    auto look = [&](int from) {
      end(from);
      steps<8>(from, [&](int g) {
#pragma unroll
        for (int i = g; i < g + 8; ++i) top = fmaxf(top, x[i]), low = fminf(low, logit(x[i], false));
      });
    };
    if (HELD) {
      look(i0);
      settle();
    } else {
      for (int from = i0; from < i1; from += AT_ONCE * kThreads) {
        fetch(from);
        look(from);
      }
    }
    return make_float2(top, low);
  }
  // Before the first pass where the range is known already, and again where the largest is infinite.
  __device__ __forceinline__ void know(bool is_infinite) {
    infinite = is_infinite;
    if (!HELD) return;
    if (infinite) fetch(i0);
    end(i0);
    settle();
  }
  // f(from): x has the logits of from + thread, from + thread + kThreads, ...
  template <typename F>
  __device__ __forceinline__ void pass(F f) {
    if (HELD) {
      f(i0);
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) asm("" : "+v"(x[i]));  // (what a pass computes of a logit is not kept in registers for the next)
    } else {
      for (int from = i0; from < i1; from += AT_ONCE * kThreads) {
        fetch(from);
        end(from);
        settle();
        f(from);
      }
    }
  }
  // f(first) for x[first .. first + STEP) up to the end
  template <int STEP, typename F>
  __device__ __forceinline__ void steps(int from, F f) {
#pragma unroll
    for (int g = 0; g < AT_ONCE; g += STEP) {
      if (from + g * kThreads >= i1) break;
      f(g);
    }
  }
  // f(logit, index) for all of a thread's, and for NaN past the end (eight at a time)
  template <typename F>
  __device__ __forceinline__ void every(F f) {
    pass([&](int from) {
      steps<8>(from, [&](int g) {
#pragma unroll
        for (int i = g; i < g + 8; ++i) f(x[i], from + static_cast<int>(threadIdx.x) + i * kThreads);
      });
    });
  }
};

// The same of a work-group's.
template <typename L>
__device__ __forceinline__ float2 range_of(RangeShared& sh, L& l) {
  const int lane = threadIdx.x & 63;
  float2 r = l.range();
  r = make_float2(wave_reduce(r.x, larger), wave_reduce(r.y, smaller));
  if (lane == 0) sh.wave_top[threadIdx.x >> 6] = r.x, sh.wave_low[threadIdx.x >> 6] = r.y;
  __syncthreads();
  return make_float2(wave_reduce(sh.wave_top[lane % kWaves], larger), wave_reduce(sh.wave_low[lane % kWaves], smaller));
}

// A row's settings, and the scale that they and its range give.
struct Settings {
  float temp, drawn, p, min_p;
  double inv;  // of the scale
  int k;
  bool by_k, by_p, by_min;
  uint64_t least;  // units that min_p asks for

  __device__ __forceinline__ Settings(const SampleArgs& a, int t)
      : temp(a.temperature ? a.temperature[t] : 1.0f),
        drawn(a.u[t]),
        p(a.top_p ? a.top_p[t] : 1.0f),
        min_p(a.min_p ? a.min_p[t] : 0.0f),
        k(a.top_k ? a.top_k[t] : 0),
        by_k(k > 0 && k < a.n),
        by_p(p < 1.0f),
        by_min(min_p > 0.0f),
        least(0) {
    inv = uniform(kPowers / kLn2 / temp);
    // (computed once: the compiler would do it again at every use)
    if (by_min) least = uniform(static_cast<uint64_t>(ceil(fmin(static_cast<double>(min_p), 1.0) * kUnit)));
  }
  __device__ __forceinline__ double number() const { return fmin(fmax(drawn, 0.0f), 0x1.fffffep-1f); }  // NaN draws as 0
  __device__ __forceinline__ double share() const { return fmax(static_cast<double>(p), 0.0); }
  __device__ __forceinline__ bool greedy(float top) const { return !(temp > 0.0f) || top == -INFINITY; }
  __device__ __forceinline__ Scale scale(const Shared& sh, float top, float low) const {
    Scale sc;
    sc.inv = inv;
    sc.top = uniform(static_cast<double>(top)), sc.half = uniform(0.5f * top);
    sc.powers = sh.powers;
    const float span = fminf(sc.half - 0.5f * low, static_cast<float>(kFar / kPowers * kLn2 / 2) * temp);
    sc.bins = uniform(span > 0.0f ? fminf((kBins - 1) / span, 3e38f) : 0.0f);  // (finite: the maximum's bin is 0)
    return sc;
  }
};

// Before the first use of a Scale and of the histogram; a barrier has to follow.
__device__ __forceinline__ void tabulate(Shared& sh) {
  if (threadIdx.x < 3) sh.found[threadIdx.x].mass = ~0ull;
  if (threadIdx.x < kPowers) sh.powers[threadIdx.x] = exp2(45 + static_cast<double>(threadIdx.x) / kPowers);
}
__device__ __forceinline__ void clear(Shared& sh) {
#pragma unroll
  for (int b = 0; b < kBins; b += kThreads) sh.mass[b + threadIdx.x] = 0, sh.count[b + threadIdx.x] = 0;
  if (threadIdx.x == 0) sh.least = 0, sh.n_list = 0, sh.n_near = 0;
}

// (The last bin's count nobody asks for, and in peaked rows most tokens are there.)
__device__ __forceinline__ void count_token(Shared& sh, int b) {
  if (b < kBins - 1) atomicAdd(&sh.count[b], 1u);
}

// The weights that min_p keeps, summed over the work-group.
__device__ __forceinline__ void keep(Shared& sh, const Settings& st, uint64_t kept) {
  if (!st.by_min) return;
  kept = wave_scan(kept);
  if ((threadIdx.x & 63) == 63 && kept) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.least), static_cast<unsigned long long>(kept));
}
__device__ __forceinline__ void add_weight(Shared& sh, int b, uint64_t w) {
  if (w) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), static_cast<unsigned long long>(w));
}

// Weighs all tokens into the histogram, two at a time: a token's chain of operations beside the
// other's.
template <bool COUNT, typename L>
__device__ __forceinline__ void weigh(Shared& sh, const Scale& sc, const Settings& st, L& l) {
  uint64_t kept = 0;
  l.pass([&](int from) {
    l.template steps<2>(from, [&](int g) {
      uint64_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = sc.weight(l.x[g + i]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int b = sc.bin(l.x[g + i]);
        if (COUNT && st.by_k) count_token(sh, b);
        add_weight(sh, b, w[i]);
      }
      if (st.by_min) {
#pragma unroll
        for (int i = 0; i < 2; ++i) kept += w[i] >= st.least ? w[i] : 0;
      }
    });
  });
  keep(sh, st, kept);
}

// The bins of the histogram in which the cuts lie.
struct Cuts {
  int k;      // the k-th token's bin, or -2
  int2 p, u;  // where top-p's and the drawn token may be, from bounds on the masses before them
  uint64_t all, from_min;

  __device__ __forceinline__ bool has(float distance) const {  // (at most a bin past the last: no weights)
    auto in = [&](int from, int to) { return distance >= from && distance < to + 1; };
    return in(k, k) || in(p.x, p.y) || in(u.x, u.y);
  }
};

// From the histogram's exclusive counts (with top-k, whose bin is bk) and its masses.
__device__ __forceinline__ Cuts cuts_of(Shared& sh, const Settings& st, int bk) {
  const Span own = scan_bins<kBins, true, false>(sh, sh.mass, sh.count, 0, 0);
  Cuts c;
  c.all = sh.all, c.from_min = st.by_min ? sh.least : c.all;
  c.k = bk;
  c.p = make_int2(-2, -2);
  const double u = st.number(), share = st.share();
  auto at = [&](int b) { return sh.mass[b]; };
  auto after = [&](int b) { return b + 1 < kBins ? at(b + 1) : c.all; };
  uint64_t lo = c.all, hi = c.all;
  if (bk >= 0) lo = at(bk), hi = after(bk);
  if (st.by_p) {
    c.p = bins_of<kBins>(sh, sh.mass, sh.count, own, limit(kReach, share * static_cast<double>(lo)),
                         limit(kReach, share * static_cast<double>(hi)));
    lo = min(lo, at(c.p.x)), hi = min(hi, after(c.p.y));
  }
  lo = min(lo, c.from_min), hi = min(hi, c.from_min);
  c.u = bins_of<kBins>(sh, sh.mass, sh.count, own, limit(kPass, u * static_cast<double>(lo)), limit(kPass, u * static_cast<double>(hi)));
  return c;
}

__device__ __forceinline__ Token token_of(const Scale& sc, float l, int at) {
  return {static_cast<uint64_t>(order_key(l)) << 32 | static_cast<uint32_t>(sc.bin(l)) << 19 | (kMostTokens - at), sc.weight(l)};
}

// Tokens whose distance a test holds for, to sh.near in any order; counts them all.
template <typename L, typename Has>
__device__ __forceinline__ void gather(Shared& sh, const Scale& sc, L& l, uint32_t* n, Has has) {
  l.pass([&](int from) {
    uint32_t mask = 0;
    l.template steps<8>(from, [&](int g) {
#pragma unroll
      for (int i = g; i < g + 8; ++i) mask |= has(sc.distance(l.x[i])) ? 1u << i : 0;
    });
    const uint32_t own = __popc(mask), upto = wave_scan(own), all = __builtin_amdgcn_readlane(upto, 63);
    if (!all) return;
    uint32_t slot = 0;
    if ((threadIdx.x & 63) == 0) slot = atomicAdd(n, all);
    slot = uniform(slot) + upto - own;
    l.template steps<8>(from, [&](int g) {
      if (!__any(mask >> g & 255)) return;
#pragma unroll
      for (int i = g; i < g + 8; ++i) {
        if (!(mask >> i & 1)) continue;
        if (slot < kList) sh.near[slot] = l.x[i], sh.near_at[slot] = from + static_cast<int>(threadIdx.x) + i * kThreads;
        ++slot;
      }
    });
  });
}

// A cut among the tokens of keys kmin to kmax, with base and rank before them, where they are more
// than the list holds (many equal logits, or an outlier that stretches the bins): the range of keys
// is divided by 1024 until one is left, then its tokens are counted.
__device__ End cut_in_range(const Limit& l, Shared& sh, Scale sc, const float* row, int n, bool infinite, uint32_t kmin, uint32_t kmax,
                            uint64_t base, uint32_t rank) {
  const int tid = threadIdx.x;
  while (kmax > kmin) {
    const int shift = max(0, 32 - __clz(kmax - kmin) - 10);
    sh.sub.mass[tid] = 0, sh.sub.count[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const float x = logit(row[i], infinite);
      const uint32_t key = order_key(x);
      if (!(x > -INFINITY) || key < kmin || key > kmax) continue;
      const uint64_t w = sc.weight(x);
      if (!w) continue;
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.sub.mass[(kmax - key) >> shift]), w);
      atomicAdd(&sh.sub.count[(kmax - key) >> shift], 1u);
    }
    __syncthreads();
    const Span own = scan_bins<kSubBins, true, true>(sh, sh.sub.mass, sh.sub.count, base, rank);
    const uint32_t b = bins_of<kSubBins>(sh, sh.sub.mass, sh.sub.count, own, l, l).x;
    base = sh.sub.mass[b], rank = sh.sub.count[b];
    kmax -= b << shift;
    kmin = max(kmin, kmax - ((1u << shift) - 1));
    __syncthreads();
  }
  // the tokens of one value, by their index: the first with enough before it
  const uint64_t w = sc.weight(key_value(kmax));
  auto& f = sh.found[l.cut];
  if (tid == 0) f.at = -1, f.mass = ~0ull;
  __syncthreads();
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + tid;
    const bool is = i < n && order_key(logit(row[i], infinite)) == kmax;
    const uint64_t votes = __ballot(is);
    if ((tid & 63) == 0) sh.wave_count[tid >> 6] = __popcll(votes);
    __syncthreads();
    uint32_t earlier = __popcll(votes & ((1ull << (tid & 63)) - 1)), every = 0;
    for (int v = 0; v < kWaves; ++v) {
      if (v < tid >> 6) earlier += sh.wave_count[v];
      every += sh.wave_count[v];
    }
    const uint64_t mass = base + earlier * w;
    if (is && !l.is_short(mass + w, rank + earlier + 1) && (l.is_short(mass, rank + earlier) || mass == 0))
      f.mass = mass + w, f.at = i;
    base += every * w, rank += every;
    __syncthreads();
    if (f.at >= 0) break;  // uniform
  }
  const End e = {f.mass, w, f.at};
  __syncthreads();
  return e;
}

// A thread's token in descending order, and what is before it in the row.
struct Place {
  uint64_t before, own;
  uint32_t rank;
  int token;
};
// Sorts the m gathered tokens of sh.order and sh.weight; earlier(slot, bin, mass, count): of the
// bins before a token's.  Changes those bins of the histogram.
template <typename Earlier>
__device__ __forceinline__ Place sorted(Shared& sh, int m, Earlier earlier) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // each counts the earlier ones, with P threads, each of which looks at every P-th
  int P = 64;
  while (P > 1 && P * m > kThreads) P /= 2;
  const int e = tid / P;
  uint32_t r = 0;
  if (e < m) {
    const uint64_t order = sh.order[e];
#pragma unroll 4
    for (int j = tid % P; j < m; j += P) r += sh.order[j] > order;
  }
  r = group_sum(r, P);
  if (e < m && tid % P == 0) sh.sorted[r] = e;
  __syncthreads();
  // thread i has the i-th: the mass before it in the list,
  const int slot = tid < m ? sh.sorted[tid] : 0;
  const uint64_t order = tid < m ? sh.order[slot] : 0, own = tid < m ? sh.weight[slot] : 0;
  const uint32_t b = static_cast<uint32_t>(order) >> 19;
  const bool leads = tid < m && (tid == 0 || static_cast<uint32_t>(sh.order[sh.sorted[tid - 1]]) >> 19 != b);
  const uint64_t upto = wave_scan(own);
  if (lane == 63) sh.wave_mass[wave] = upto;
  __syncthreads();
  uint64_t before = row_sum(lane % kWaves < wave ? sh.wave_mass[lane % kWaves] : 0) + upto - own;
  // and in the row, from where the first of its bin is
  if (leads) {
    uint64_t mass;
    uint32_t count;
    earlier(slot, b, mass, count);
    sh.mass[b] = mass - before, sh.count[b] = count - tid;
  }
  __syncthreads();
  return {before + sh.mass[b], own, tid + sh.count[b], kMostTokens - static_cast<int>(order & kMostTokens)};
}

// A cut among them: each knows what is before it, and one of them is the end (own is 0 for
// threads without one).
__device__ __forceinline__ End cut_in_list(const Limit& l, Shared& sh, const Place& p) {
  auto& f = sh.found[l.cut];  // as tabulate() left it where none is: all are kept
  if (p.own && !l.is_short(p.before + p.own, p.rank + 1) && (l.is_short(p.before, p.rank) || p.before == 0))
    f.mass = p.before + p.own, f.weight = p.own, f.at = p.token;
  __syncthreads();
  return {f.mass, f.weight, f.at};
}

// A cut by the exclusive sums of all bins and the tokens of the one that it lies in.
template <typename L>
__device__ __forceinline__ End cut_in_bin(const Limit& limit, Shared& sh, const Scale& sc, L& l, int n) {
  const int tid = threadIdx.x;
  for (int b = tid; b < kBins; b += kThreads) {
    if ((b == 0 || limit.is_short(sh.mass[b], sh.count[b])) &&
        (b == kBins - 1 || !limit.is_short(sh.mass[b + 1], sh.count[b + 1])))
      sh.found_bin[limit.cut][0] = b;
  }
  if (tid == 0) sh.n_list = 0, sh.key_low = ~0u, sh.key_top = 0;
  __syncthreads();
  const int b = sh.found_bin[limit.cut][0];
  const uint64_t mass = sh.mass[b];
  const uint32_t count = sh.count[b];
  auto in = [&](float d) { return d >= b && d < b + 1; };
  gather(sh, sc, l, &sh.n_list, in);
  __syncthreads();
  const int m = static_cast<int>(sh.n_list);
  if (m <= kList) {
    if (tid < m) {
      const Token x = token_of(sc, sh.near[tid], sh.near_at[tid]);
      sh.order[tid] = x.order, sh.weight[tid] = x.weight;
    }
    __syncthreads();
    const Place p = sorted(sh, m, [&](int, uint32_t, uint64_t& x, uint32_t& y) { x = mass, y = count; });
    const End e = cut_in_list(limit, sh, p);
    if (tid == 0) sh.mass[b] = mass, sh.count[b] = count;
    __syncthreads();
    return e;
  }
  uint32_t low = ~0u, top = 0;
  l.every([&](float x, int) {
    if (!in(sc.distance(x))) return;
    low = min(low, order_key(x)), top = max(top, order_key(x));
  });
  if (top) atomicMin(&sh.key_low, low), atomicMax(&sh.key_top, top);
  __syncthreads();
  return cut_in_range(limit, sh, sc, l.row, n, l.infinite, sh.key_low, sh.key_top, mass, count);
}

// The choice among the m gathered tokens of sh.order and sh.weight; where there are more than the
// list holds, cut by cut, with the exclusive sums that all() leaves in the histogram.
template <typename Earlier, typename All>
__device__ __forceinline__ void choose(Shared& sh, const SampleArgs& a, const Settings& st, const Scale& sc, bool infinite, int t, int m,
                                       uint64_t whole, uint64_t from_min, Earlier earlier, All all) {
  const double u = st.number(), share = st.share();
  uint64_t M = whole;
  End end;
  if (m <= kList) {
    const Place p = sorted(sh, m, earlier);
    if (st.by_k) M = min(M, cut_in_list(limit(kCount, st.k), sh, p).mass);
    if (st.by_p) M = min(M, cut_in_list(limit(kReach, share * static_cast<double>(M)), sh, p).mass);
    M = min(M, from_min);
    end = cut_in_list(limit(kPass, u * static_cast<double>(M)), sh, p);
  } else {
    all();
    Logits<kRead> l(a.logits + static_cast<size_t>(t) * a.n, 0, a.n);
    l.know(infinite);
#pragma unroll 1
    for (int c = st.by_k ? kCount : st.by_p ? kReach : kPass; c <= kPass; ++c) {
      if (c == kReach && !st.by_p) continue;
      if (c == kPass) M = min(M, from_min);
      end = cut_in_bin(limit(static_cast<Cut>(c), c == kCount ? st.k : (c == kReach ? share : u) * static_cast<double>(M)), sh, sc, l, a.n);
      if (c < kPass) M = min(M, end.mass);
    }
  }
  if (threadIdx.x == 0) {
    a.idx[t] = end.token;
    if (a.prob) a.prob[t] = static_cast<float>(static_cast<double>(end.weight) / static_cast<double>(M));
  }
}

// A work-group per row, its logits in registers up to 32768.  Bound by the instructions of the
// weights, some thirty a token of which half are in double precision, and by a chain of scans and
// barriers: with top-k, or min-p alone, only the tokens down to a cut's bin are weighed, from a
// list.  One row of 32000: 13.3 us with top-k of 50, 18 with all tokens (8 of them weights);
// 500 rows with min-p: 26.5 us, 2.4 TB/s, in two rounds of work-groups (128 registers: one a CU).
template <int AT_ONCE>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int t = blockIdx.x, tid = threadIdx.x;
  Logits<AT_ONCE> l(a.logits + static_cast<size_t>(t) * a.n, 0, a.n);
  const Settings st(a, t);
  tabulate(sh);
  clear(sh);
  if (tid == 0) sh.at = a.n;
  float2 r = range_of(sh, l);
  if (r.x == INFINITY) l.know(true), r = make_float2(0.0f, 0.0f);
  if (st.greedy(r.x)) {
    int at = a.n;
    l.every([&](float x, int i) { at = x == r.x && i < at ? i : at; });
    if (at < a.n) atomicMin(&sh.at, at);
    __syncthreads();
    if (tid == 0) {
      a.idx[t] = r.x > -INFINITY ? sh.at : 0;
      if (a.prob) a.prob[t] = 1.0f;
    }
    return;
  }
  const Scale sc = st.scale(sh, r.x, r.y);
  int last = kBins - 1;  // the last bin that matters
  if (st.by_min && !st.by_p) {  // of the least weight that rounds up to min_p's units (a bin further, for its fp32 distances)
    const double w = (static_cast<double>(st.least) - 0.5) / kUnit;
    const float far = fmaxf(-logf(static_cast<float>(w)), static_cast<float>(1.0 - w));  // (next to 1 the logarithm gives 0)
    last = static_cast<int>(fminf(far * st.temp * 0.500005f * sc.bins, kBins - 2)) + 1;
  }
  if (st.by_k) {
    l.every([&](float x, int) { count_token(sh, sc.bin(x)); });
    __syncthreads();
    const Span own = scan_bins<kBins, false, true>(sh, sh.mass, sh.count, 0, 0);
    last = min(last, bins_of<kBins>(sh, sh.mass, sh.count, own, limit(kCount, st.k), limit(kCount, st.k)).x);
  }
  bool few = last < kBins - 1 && !(st.by_k && sh.count[last + 1] > kList);
  if (few) {
    gather(sh, sc, l, &sh.n_near, [&](float d) { return d < last + 1; });
    __syncthreads();
    few = sh.n_near <= kList;
  }
  Token own = {};
  if (few) {
    if (tid < static_cast<int>(sh.n_near)) {
      own = token_of(sc, sh.near[tid], sh.near_at[tid]);
      add_weight(sh, sc.bin(sh.near[tid]), own.weight);
    }
    keep(sh, st, own.weight >= st.least ? own.weight : 0);
  } else {
    weigh<false>(sh, sc, st, l);
  }
  __syncthreads();
  const Cuts c = cuts_of(sh, st, st.by_k ? last : -2);  // (a bin before the k-th token's where min_p ends there)
  if (few) {
    if (own.weight && c.has(sc.distance(sh.near[tid]))) {
      const uint32_t slot = atomicAdd(&sh.n_list, 1u);
      sh.order[slot] = own.order, sh.weight[slot] = own.weight;
    }
  } else {
    gather(sh, sc, l, &sh.n_list, [&](float d) { return c.has(d); });
    __syncthreads();
    if (tid < static_cast<int>(min(sh.n_list, static_cast<uint32_t>(kList)))) {
      own = token_of(sc, sh.near[tid], sh.near_at[tid]);
      sh.order[tid] = own.order, sh.weight[tid] = own.weight;
    }
  }
  __syncthreads();
  choose(sh, a, st, sc, l.infinite, t, static_cast<int>(sh.n_list), c.all, c.from_min,
         [&](int, uint32_t b, uint64_t& mass, uint32_t& count) { mass = sh.mass[b], count = sh.count[b]; }, [] {});
}

// The same by several work-groups a row, in four launches: the range of each, one histogram of
// them all, the tokens of the cuts' bins, and the choice.  64 rows of 131071 logits: 7.4, 18.2, 12.9
// and 5.2 us.  (A histogram for each work-group, summed by the next launch, instead of atomics: the
// same; the last of a row's work-groups to choose instead of a fourth launch: as long, as its fence
// waits for the L2.)
struct Gathered {
  Token token;
  uint64_t mass;  // of the bins before
  uint64_t count;
};
struct SplitRow {  // a row's part of the workspace
  uint64_t mass[kBins];
  uint32_t count[kBins];
  Gathered list[kList];
  float2 range[kCus];
  uint64_t least, all;
  uint32_t n_list;
  int32_t at;  // of the arg max

  __device__ __forceinline__ float2 whole(int splits) const {
    const int i = threadIdx.x & 63;
    float top = -INFINITY, low = INFINITY;
    for (int s = i; s < splits; s += 64) top = fmaxf(top, range[s].x), low = fminf(low, range[s].y);
    return make_float2(wave_reduce(top, larger), wave_reduce(low, smaller));
  }
};
__device__ __forceinline__ SplitRow& split_row(const SampleArgs& a, int t) { return static_cast<SplitRow*>(a.workspace)[t]; }
template <int AT_ONCE>
__device__ __forceinline__ Logits<AT_ONCE> share_of(const SampleArgs& a, int s, int t) {
  return Logits<AT_ONCE>(a.logits + static_cast<size_t>(t) * a.n, min(s * a.share, a.n), min((s + 1) * a.share, a.n));
}

// A work-group's part and row.  Work-groups go to the 8 XCDs in turn, and a row's stay on one: its
// L2 has what the launch before read and what the others wrote.
struct Part {
  int s, t;
};
__device__ __forceinline__ Part part_of(const SampleArgs& a) {
  const int i = blockIdx.x / kXcds;
  return {i % a.splits, i / a.splits * kXcds + static_cast<int>(blockIdx.x % kXcds)};
}

template <int AT_ONCE>
__global__ __launch_bounds__(kThreads) void sample_range_kernel(SampleArgs a) {
  __shared__ RangeShared sh;
  const auto [s, t] = part_of(a);
  if (t >= a.T) return;
  SplitRow& ws = split_row(a, t);
  Logits<AT_ONCE> l = share_of<AT_ONCE>(a, s, t);
  for (int b = s * kThreads + static_cast<int>(threadIdx.x); b < kBins; b += a.splits * kThreads) ws.mass[b] = 0, ws.count[b] = 0;
  if (s == 0 && threadIdx.x == 0) ws.least = 0, ws.n_list = 0, ws.at = a.n;
  const float2 r = range_of(sh, l);
  if (threadIdx.x == 0) ws.range[s] = r;
}

template <int AT_ONCE>
__global__ __launch_bounds__(kThreads) void sample_weigh_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const auto [s, t] = part_of(a);
  const int tid = threadIdx.x;
  if (t >= a.T) return;
  SplitRow& ws = split_row(a, t);
  Logits<AT_ONCE> l = share_of<AT_ONCE>(a, s, t);
  const Settings st(a, t);
  tabulate(sh);
  clear(sh);
  float2 r = ws.whole(a.splits);
  l.know(r.x == INFINITY);
  if (l.infinite) r = make_float2(0.0f, 0.0f);
  if (st.greedy(r.x)) {
    int at = a.n;
    l.every([&](float x, int i) { at = x == r.x && i < at ? i : at; });
    if (at < a.n && r.x > -INFINITY) atomicMin(&ws.at, at);
    return;
  }
  const Scale sc = st.scale(sh, r.x, r.y);
  __syncthreads();
  weigh<true>(sh, sc, st, l);
  __syncthreads();
#pragma unroll
  for (int b = 0; b < kBins; b += kThreads) {
    if (const uint64_t x = sh.mass[b + tid]) atomicAdd(reinterpret_cast<unsigned long long*>(ws.mass + b + tid), x);
    if (const uint32_t x = sh.count[b + tid]) atomicAdd(ws.count + b + tid, x);
  }
  if (tid == 0 && sh.least) atomicAdd(reinterpret_cast<unsigned long long*>(&ws.least), sh.least);
}

template <int AT_ONCE>
__global__ __launch_bounds__(kThreads) void sample_gather_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const auto [s, t] = part_of(a);
  const int tid = threadIdx.x;
  if (t >= a.T) return;
  SplitRow& ws = split_row(a, t);
  Logits<AT_ONCE> l = share_of<AT_ONCE>(a, s, t);
  const Settings st(a, t);
#pragma unroll
  for (int b = 0; b < kBins; b += kThreads) sh.mass[b + tid] = ws.mass[b + tid], sh.count[b + tid] = ws.count[b + tid];
  if (tid == 0) sh.least = ws.least, sh.n_list = 0;
  tabulate(sh);
  float2 r = ws.whole(a.splits);
  l.know(r.x == INFINITY);
  if (l.infinite) r = make_float2(0.0f, 0.0f);
  if (st.greedy(r.x)) return;
  const Scale sc = st.scale(sh, r.x, r.y);
  __syncthreads();
  int bk = -2;
  if (st.by_k) {
    const Span own = scan_bins<kBins, false, true>(sh, sh.mass, sh.count, 0, 0);
    bk = bins_of<kBins>(sh, sh.mass, sh.count, own, limit(kCount, st.k), limit(kCount, st.k)).x;
  }
  const Cuts c = cuts_of(sh, st, bk);
  gather(sh, sc, l, &sh.n_list, [&](float d) { return c.has(d); });
  __syncthreads();
  const uint32_t m = sh.n_list;
  if (tid == 0) sh.at = static_cast<int32_t>(atomicAdd(&ws.n_list, m));
  __syncthreads();
  const uint32_t slot = static_cast<uint32_t>(sh.at) + tid;
  if (tid < static_cast<int>(m) && slot < kList) {
    const Token x = token_of(sc, sh.near[tid], sh.near_at[tid]);
    const uint32_t b = static_cast<uint32_t>(x.order) >> 19;
    ws.list[slot] = {x, sh.mass[b], sh.count[b]};
  }
  if (s == 0 && tid == 0) ws.all = c.all;
}

__global__ __launch_bounds__(kThreads) void sample_choose_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int t = blockIdx.x, tid = threadIdx.x;
  const SplitRow& ws = split_row(a, t);
  const Settings st(a, t);
  tabulate(sh);
  float2 r = ws.whole(a.splits);
  const bool infinite = r.x == INFINITY;
  if (infinite) r = make_float2(0.0f, 0.0f);
  if (st.greedy(r.x)) {
    if (tid == 0) {
      a.idx[t] = r.x > -INFINITY ? ws.at : 0;
      if (a.prob) a.prob[t] = 1.0f;
    }
    return;
  }
  const int m = static_cast<int>(ws.n_list);
  if (m <= kList && tid < m) sh.order[tid] = ws.list[tid].token.order, sh.weight[tid] = ws.list[tid].token.weight;
  __syncthreads();
  const Scale sc = st.scale(sh, r.x, r.y);
  choose(sh, a, st, sc, infinite, t, m, ws.all, st.by_min ? ws.least : ws.all,
         [&](int e, uint32_t, uint64_t& mass, uint32_t& count) { mass = ws.list[e].mass, count = static_cast<uint32_t>(ws.list[e].count); },
         [&] {
           for (int b = tid; b < kBins; b += kThreads) sh.mass[b] = ws.mass[b], sh.count[b] = ws.count[b];
           __syncthreads();
           scan_bins<kBins, true, true>(sh, sh.mass, sh.count, 0, 0);
         });
}

// Work-groups of a row: as many as leave one a CU of the XCD that the row's are on, of at least
// kLeastShare logits each; but one where that saves it fewer than 40000 logits, which take
// as long as three more launches, or where only two or three would do, whose merged histograms
// cost what they save.  One | several, us, from top-k of 50 to all tokens: one row of 32000
// 14-20 | 21-24, of 50257 24-33 | 21-24, of 131071 42-66 | 22-25; 64 rows of 50257 23-32 | 29-33, of
// 131071 45-70 | 40-45; 128 rows of 131071 46-72 | 64-68.
constexpr int kLeastShare = 4096;
int splits_of(int T, int n) {
  const int rows = (std::max(T, 1) - 1) / kXcds + 1;  // of an XCD
  const int splits = std::min(kCus / kXcds / rows, n / kLeastShare);
  return splits < 4 || n - n / splits < 40000 ? 1 : splits;
}

}  // namespace

extern "C" {

ms_status ms_sample_workspace(int32_t T, int32_t n, uint64_t* bytes_out) {
  if (T < 0 || n <= 0 || !bytes_out) return MS_E_INVALID;
  if (n > kMostTokens) return MS_E_UNSUPPORTED;
  const int splits = splits_of(T, n);
  *bytes_out = splits > 1 ? T * sizeof(SplitRow) : 0;
  return MS_OK;
}

ms_status ms_sample(const float* logits, int32_t T, int32_t n, const ms_sample_opts* opts, const float* u_dev,
                    int32_t* idx_out, float* prob_out, void* workspace_dev, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (const ms_status st = ms_sample_workspace(T, n, &need); st != MS_OK) return st;
  if (T == 0) return MS_OK;
  if (!logits || !u_dev || !idx_out) return MS_E_INVALID;
  if (need > 0 && (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15u) || workspace_bytes < need))
    return MS_E_INVALID;
  const size_t values = 4 * static_cast<size_t>(T);
  const ms_sample_opts given = opts ? *opts : ms_sample_opts{};
  auto apart = [&](const void* o, size_t bytes) {  // from all inputs
    const void* const rows[] = {u_dev, given.temperature_dev, given.top_k_dev, given.top_p_dev, given.min_p_dev};
    return std::none_of(std::begin(rows), std::end(rows), [&](const void* q) { return overlap(o, bytes, q, values); }) &&
           !overlap(o, bytes, logits, values * n);
  };
  if (!apart(idx_out, values) || !apart(prob_out, values) || overlap(idx_out, values, prob_out, values)) return MS_E_INVALID;
  // (the workspace is written before inputs are read for the last time)
  if (need > 0 && (!apart(workspace_dev, need) || overlap(workspace_dev, need, idx_out, values) ||
                   overlap(workspace_dev, need, prob_out, values)))
    return MS_E_INVALID;
  if (T > UINT32_MAX / kThreads) return MS_E_UNSUPPORTED;
  const int splits = splits_of(T, n);
  const SampleArgs a = {logits, u_dev, given.temperature_dev, given.top_p_dev, given.min_p_dev, given.top_k_dev, idx_out, prob_out,
                        T, n, splits, (n - 1) / splits + 1, workspace_dev};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 rows(static_cast<unsigned>(T)), all((static_cast<unsigned>(T) + kXcds - 1) / kXcds * kXcds * splits), block(kThreads);
  auto launch = [&](auto at_once) {
    constexpr int AT_ONCE = decltype(at_once)::value;
    if (splits == 1) {
      hipLaunchKernelGGL(sample_kernel<AT_ONCE>, rows, block, 0, s, a);
    } else {
      hipLaunchKernelGGL(sample_range_kernel<AT_ONCE>, all, block, 0, s, a);
      hipLaunchKernelGGL(sample_weigh_kernel<AT_ONCE>, all, block, 0, s, a);
      hipLaunchKernelGGL(sample_gather_kernel<AT_ONCE>, all, block, 0, s, a);
      hipLaunchKernelGGL(sample_choose_kernel, rows, block, 0, s, a);
    }
  };
  if (a.share <= kHold * kThreads) launch(std::integral_constant<int, kHold>());
  else launch(std::integral_constant<int, kRead>());
  return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP;
}

}  // extern "C"
