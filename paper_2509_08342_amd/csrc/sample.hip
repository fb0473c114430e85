// A token drawn from each row of logits: temperature, top-k, top-p and min-p, from given
// random numbers.  Stateless, like the other calls of the decoder loop.
//
// With the logits l in descending order, ties to the lower index, and weights
// exp((l - max) / temperature), every filter keeps a prefix, so the kept mass M is the least
// of the filters' masses, and the token is the first whose running mass passes u M: top-k
// keeps the mass of the first k, top-p of the fewest that reach p of that, min-p of the weights
// from min-p on.  No row
// is sorted: a histogram over the distance from the maximum gives the running mass at 8192
// borders; only the tokens of the few bins in which a filter or the drawn mass ends are
// gathered, and each of them finds its own running mass by comparing itself with the others.
//
// Weights are whole numbers of 2^-45, computed in double precision: their sums do not depend
// on the order of additions (so atomics may build them), and a border between two tokens is
// off by 2^-46 of the largest weight per token before it, where fp32 sums of 10^5 tokens
// would move it by more than the smallest tokens' weights.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kernels.h"
#include "moesplit.h"

namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 8192;
constexpr int kList = kThreads;  // gathered tokens
constexpr int kSubBins = 1024;   // of rows whose tokens crowd into few bins
constexpr int kMostTokens = (1 << 19) - 1;  // n 2^45 < 2^64
constexpr double kUnit = 35184372088832.0;  // 2^45
constexpr int kCus = 256, kXcds = 8;
constexpr double kFar = 46 * 256;  // 2^-46 rounds to zero units (in 256ths of powers of two)
constexpr int kHold = 32;          // logits of a thread in registers at a time

// A logit as it counts: NaN as -infinity; where the largest is infinite, its likes are 0 and all
// others -infinity.
__device__ __forceinline__ float logit(float x, bool infinite) {
  if (infinite) x = x == INFINITY ? 0.0f : -INFINITY;
  return x == x ? x : -INFINITY;
}

// order of fp32 values as unsigned numbers; -0 and 0 alike
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// What a row's tokens are weighed with.
constexpr int kPowers = 256;
struct Scale {
  double inv;   // kPowers / (ln 2 temperature)
  float top;    // the largest logit (finite)
  float bins;   // per unit of logits
  const double* powers;  // 2^(-i / kPowers)

  // by the distance from the maximum in fp32: never less for a smaller logit
  __device__ __forceinline__ int bin(float l) const { return static_cast<int>(fminf((top - l) * bins, kBins - 1)); }
  // exp((l - top) / temperature) in units: 2^(-j / kPowers) from the table and the series of the
  // rest, |r| <= 1/2, to its fourth power (the next term is 2^-54)
  __device__ __forceinline__ uint64_t weight(float l) const {
    const double y = fmin((static_cast<double>(top) - l) * inv, kFar + kPowers);  // (NaN, of an endless temperature, too)
    constexpr double L = 0.69314718055994530942 / kPowers;
    const double j = rint(y), r = y - j;
    double s = fma(r, L * L * L * L / 24, -L * L * L / 6);
    s = fma(r, s, L * L / 2);
    s = fma(r, s, -L);
    s = fma(r, s, 1.0);
    const int i = static_cast<int>(j);
    const double e = s * powers[i & (kPowers - 1)];
    const long long scaled = __double_as_longlong(e) + (static_cast<long long>(45 - i / kPowers) << 52);
    // rounds to a whole number in the low bits
    return static_cast<uint64_t>(__double_as_longlong(__longlong_as_double(scaled) + 4503599627370496.0)) & ((1ull << 52) - 1);
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

struct Shared {
  uint64_t mass[kBins];   // then exclusive sums
  uint32_t count[kBins];
  union {
    Token list[kList];
    struct {
      uint64_t mass[kSubBins];
      uint32_t count[kSubBins];
    } sub;
  };
  double powers[kPowers];
  uint64_t wave_mass[kThreads / 64];
  uint32_t wave_count[kThreads / 64];
  float wave_top[kThreads / 64], wave_low[kThreads / 64];
  int32_t wave_at[kThreads / 64];
  uint64_t all, least, found_mass, found_weight;
  uint32_t all_count, n_list;
  int32_t found_at, found_bin[2];
};

// Bin b's place: a thread's bins, which follow each other, lie kThreads apart.
template <int BINS>
__device__ __forceinline__ int place(int b) {
  constexpr unsigned PER = BINS / kThreads;
  return static_cast<unsigned>(b) % PER * kThreads + static_cast<unsigned>(b) / PER;
}

// Exclusive sums of mass and count in place; the totals to sh.all and sh.all_count.  Returns
// the sums before and behind the thread's own bins.
struct Span {
  uint64_t mass0, mass1;
  uint32_t count0, count1;
};
template <int BINS, bool MASS, bool COUNT>
__device__ __forceinline__ Span scan_bins(Shared& sh, uint64_t* mass, uint32_t* count, uint64_t mass0, uint32_t count0) {
  constexpr int PER = BINS / kThreads, WAVES = kThreads / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t m = 0;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (MASS) m += mass[i * kThreads + tid];
    if (COUNT) c += count[i * kThreads + tid];
  }
  uint64_t im = m;
  uint32_t ic = c;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint64_t om = MASS ? __shfl_up(static_cast<unsigned long long>(im), s, 64) : 0;
    const uint32_t oc = COUNT ? __shfl_up(ic, s, 64) : 0;
    if (lane >= s) im += om, ic += oc;
  }
  if (lane == 63) sh.wave_mass[wave] = im, sh.wave_count[wave] = ic;
  __syncthreads();
  uint64_t wm = MASS && lane < WAVES && lane < wave ? sh.wave_mass[lane] : 0;  // of the waves before
  uint32_t wc = COUNT && lane < WAVES && lane < wave ? sh.wave_count[lane] : 0;
#pragma unroll
  for (int s = WAVES / 2; s >= 1; s >>= 1) {
    if (MASS) wm += __shfl_xor(static_cast<unsigned long long>(wm), s, 64);
    if (COUNT) wc += __shfl_xor(wc, s, 64);
  }
  uint64_t base = mass0 + __shfl(static_cast<unsigned long long>(wm), 0, 64) + im - m;
  uint32_t bc = count0 + __shfl(wc, 0, 64) + ic - c;
  const Span own = {base, base + m, bc, bc + c};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = i * kThreads + tid;
    if (MASS) {
      const uint64_t x = mass[at];
      mass[at] = base;
      base += x;
    }
    if (COUNT) {
      const uint32_t y = count[at];
      count[at] = bc;
      bc += y;
    }
  }
  if (tid == kThreads - 1) {
    if (MASS) sh.all = base;
    if (COUNT) sh.all_count = bc;
  }
  __syncthreads();
  return own;
}

// Where a prefix ends: at the token that makes it t long, that takes its mass to t, or past t.
enum Cut { kCount, kReach, kPass };

// Whether the prefix before `mass` and `count` is still short of the cut.
template <Cut CUT>
__device__ __forceinline__ bool is_short(double t, uint64_t mass, uint32_t count) {
  return CUT == kCount ? count < t : CUT == kReach ? static_cast<double>(mass) < t : static_cast<double>(mass) <= t;
}

// The bins in which the cuts at t0 and t1 lie, from exclusive sums: of the threads whose bins
// they may be in exactly one looks (the last where rounding leaves none).
template <Cut CUT, int BINS>
__device__ __forceinline__ int2 bins_of(Shared& sh, const uint64_t* mass, const uint32_t* count, const Span& own, double t0, double t1) {
  constexpr int PER = BINS / kThreads;
  const int tid = threadIdx.x;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const double t = i ? t1 : t0;
    if ((tid == 0 || is_short<CUT>(t, own.mass0, own.count0)) && (tid == kThreads - 1 || !is_short<CUT>(t, own.mass1, own.count1))) {
      int b = tid * PER;
#pragma unroll
      for (int j = 1; j < PER; ++j)
        if (is_short<CUT>(t, mass[j * kThreads + tid], count[j * kThreads + tid])) b = tid * PER + j;
      sh.found_bin[i] = b;
    }
  }
  __syncthreads();
  const int2 r = make_int2(sh.found_bin[0], sh.found_bin[1]);
  __syncthreads();
  return r;
}

struct End {
  uint64_t mass, weight;  // of the prefix, the token at its end included, and of that token
  int token;
};

// A cut among the gathered tokens: each knows what is before it, and one of them is the end
// (own is 0 for threads without one).
template <Cut CUT>
__device__ __forceinline__ End cut_in_list(Shared& sh, double t, uint64_t before, uint32_t rank, uint64_t own, int token) {
  if (threadIdx.x == 0) sh.found_mass = ~0ull;  // none: all are kept
  __syncthreads();
  if (own && !is_short<CUT>(t, before + own, rank + 1) && (is_short<CUT>(t, before, rank) || before == 0))
    sh.found_mass = before + own, sh.found_weight = own, sh.found_at = token;
  __syncthreads();
  const End e = {sh.found_mass, sh.found_weight, sh.found_at};
  __syncthreads();
  return e;
}

// The same for rows whose tokens crowd into few bins (many equal logits, or an outlier that
// stretches the bins): the range of values is divided by 1024 until one value is left, then
// its tokens are counted.
template <Cut CUT>
__device__ End cut_in_row(Shared& sh, Scale sc, const float* row, int n, bool infinite, float low, double t) {
  const int tid = threadIdx.x;
  uint32_t kmax = order_key(sc.top), kmin = order_key(low);
  uint64_t base = 0;
  uint32_t rank = 0;
  while (kmax > kmin) {
    const int shift = max(0, 32 - __clz(kmax - kmin) - 10);
    sh.sub.mass[tid] = 0, sh.sub.count[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const float l = logit(row[i], infinite);
      const uint32_t key = order_key(l);
      if (!(l > -INFINITY) || key < kmin || key > kmax) continue;
      const uint64_t w = sc.weight(l);
      if (!w) continue;
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.sub.mass[(kmax - key) >> shift]), w);
      atomicAdd(&sh.sub.count[(kmax - key) >> shift], 1u);
    }
    __syncthreads();
    const Span own = scan_bins<kSubBins, true, true>(sh, sh.sub.mass, sh.sub.count, base, rank);
    const uint32_t b = bins_of<CUT, kSubBins>(sh, sh.sub.mass, sh.sub.count, own, t, t).x;
    base = sh.sub.mass[b], rank = sh.sub.count[b];
    kmax -= b << shift;
    kmin = max(kmin, kmax - ((1u << shift) - 1));
    __syncthreads();
  }
  // the tokens of one value, by their index: the first with enough before it
  const uint64_t w = sc.weight(key_value(kmax));
  if (tid == 0) sh.found_at = -1, sh.found_mass = ~0ull;
  __syncthreads();
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + tid;
    const bool is = i < n && order_key(logit(row[i], infinite)) == kmax;
    const uint64_t votes = __ballot(is);
    if ((tid & 63) == 0) sh.wave_count[tid >> 6] = __popcll(votes);
    __syncthreads();
    uint32_t earlier = __popcll(votes & ((1ull << (tid & 63)) - 1)), every = 0;
    for (int v = 0; v < kThreads / 64; ++v) {
      if (v < tid >> 6) earlier += sh.wave_count[v];
      every += sh.wave_count[v];
    }
    const uint64_t mass = base + earlier * w;
    if (is && !is_short<CUT>(t, mass + w, rank + earlier + 1) && (is_short<CUT>(t, mass, rank + earlier) || mass == 0))
      sh.found_mass = mass + w, sh.found_at = i;
    base += every * w, rank += every;
    __syncthreads();
    if (sh.found_at >= 0) break;  // uniform
  }
  const End e = {sh.found_mass, w, sh.found_at};
  __syncthreads();
  return e;
}

// A thread's logits of [i0, i1) of a row, read kHold at a time, and only once where there are no
// more.
struct Logits {
  const float* row;
  int i0, i1;
  bool infinite;
  float hold[kHold];

  __device__ __forceinline__ bool once() const { return i1 - i0 <= kHold * kThreads; }
  __device__ __forceinline__ void fetch(int from) {  // from + thread, from + thread + kThreads, ...
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int j = from + static_cast<int>(threadIdx.x) + i * kThreads;
      hold[i] = j < i1 ? row[j] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < kHold; ++i) hold[i] = logit(hold[i], infinite);
  }
  __device__ __forceinline__ Logits(const float* r, int from, int to) : row(r), i0(from), i1(to), infinite(false) {
    if (once()) fetch(i0);
  }
  __device__ __forceinline__ void make_infinite() {
    infinite = true;
    if (once()) {
#pragma unroll
      for (int i = 0; i < kHold; ++i) hold[i] = logit(hold[i], true);
    }
  }
  // f(logit, index) for the thread's, and for -infinity past the end (eight at a time)
  template <typename F>
  __device__ __forceinline__ void every(F f) {
    for (int from = i0; from < i1; from += kHold * kThreads) {
      if (!once()) fetch(from);
#pragma unroll
      for (int g = 0; g < kHold; g += 8) {
        if (from + g * kThreads >= i1) break;
#pragma unroll
        for (int i = g; i < g + 8; ++i) f(hold[i], from + static_cast<int>(threadIdx.x) + i * kThreads);
      }
    }
  }
  // f(four logits)
  template <typename F>
  __device__ __forceinline__ void fours(F f) {
    for (int from = i0; from < i1; from += kHold * kThreads) {
      if (!once()) fetch(from);
#pragma unroll
      for (int g = 0; g < kHold; g += 4) {
        if (from + g * kThreads >= i1) break;
        const float x[4] = {hold[g], hold[g + 1], hold[g + 2], hold[g + 3]};
        f(x);
      }
    }
  }
};

// The largest and the smallest of a work-group's logits.
__device__ __forceinline__ float2 range_of(Shared& sh, Logits& l) {
  constexpr int WAVES = kThreads / 64;
  const int lane = threadIdx.x & 63;
  float top = -INFINITY, low = INFINITY;
  l.every([&](float x, int) { top = fmaxf(top, x), low = fminf(low, x); });
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64)), low = fminf(low, __shfl_xor(low, s, 64));
  if (lane == 0) sh.wave_top[threadIdx.x >> 6] = top, sh.wave_low[threadIdx.x >> 6] = low;
  __syncthreads();
  top = sh.wave_top[lane % WAVES], low = sh.wave_low[lane % WAVES];
#pragma unroll
  for (int s = WAVES / 2; s >= 1; s >>= 1)
    top = fmaxf(top, __shfl_xor(top, s, 64)), low = fminf(low, __shfl_xor(low, s, 64));
  return make_float2(top, low);
}

// A row's settings, and the scale that they and its range give.
struct Settings {
  float temp, drawn, p, min_p;
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
        least(by_min ? static_cast<uint64_t>(ceil(fmin(static_cast<double>(min_p), 1.0) * kUnit)) : 0) {}
  __device__ __forceinline__ double number() const { return fmin(fmax(drawn, 0.0f), 0x1.fffffep-1f); }  // NaN draws as 0
  __device__ __forceinline__ double share() const { return fmax(static_cast<double>(p), 0.0); }
  __device__ __forceinline__ bool greedy(float top) const { return !(temp > 0.0f) || top == -INFINITY; }
  __device__ __forceinline__ Scale scale(const Shared& sh, float top, float low) const {
    constexpr double kLn2 = 0.69314718055994530942;
    Scale sc;
    sc.inv = kPowers / kLn2 / temp;
    sc.top = top;
    sc.powers = sh.powers;
    const float span = fminf(top - low, static_cast<float>(kFar / kPowers * kLn2) * temp);
    sc.bins = span > 0.0f ? fminf((kBins - 1) / span, 3e38f) : 0.0f;  // (finite: the maximum's bin is 0)
    return sc;
  }
};

// Before the first use of a Scale and of the histogram; a barrier has to follow.
__device__ __forceinline__ void tabulate(Shared& sh) {
  if (threadIdx.x < kPowers) sh.powers[threadIdx.x] = exp2(-static_cast<double>(threadIdx.x) / kPowers);
}
__device__ __forceinline__ void clear(Shared& sh) {
#pragma unroll
  for (int b = 0; b < kBins; b += kThreads) sh.mass[b + threadIdx.x] = 0, sh.count[b + threadIdx.x] = 0;
  if (threadIdx.x == 0) sh.least = 0;
}

// (The last bin's count nobody asks for, and in peaked rows most tokens are there.)
__device__ __forceinline__ void count_token(Shared& sh, int b) {
  if (b < kBins - 1) atomicAdd(&sh.count[place<kBins>(b)], 1u);
}

// Weighs the tokens of bins 0 .. last into the histogram, and sums those that min_p keeps.
template <bool COUNT>
__device__ __forceinline__ void weigh(Shared& sh, const Scale& sc, const Settings& st, Logits& l, int last) {
  uint64_t kept = 0;
  auto add = [&](int b, uint64_t w) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[place<kBins>(b)]), w);
    kept += w >= st.least ? w : 0;
  };
  if (last < kBins - 1) {  // few
    l.every([&](float x, int) {
      const int b = sc.bin(x);
      if (b > last) return;
      if (const uint64_t w = sc.weight(x)) add(b, w);
    });
  } else {
    l.fours([&](const float (&x)[4]) {  // a token's chain of operations beside the others'
      uint64_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = sc.weight(x[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = sc.bin(x[i]);
        if (COUNT && st.by_k) count_token(sh, b);
        if (w[i]) add(b, w[i]);
      }
    });
  }
  if (st.by_min) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) kept += __shfl_xor(static_cast<unsigned long long>(kept), s, 64);
    if ((threadIdx.x & 63) == 0) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.least), static_cast<unsigned long long>(kept));
  }
}

// The bins of the histogram in which the cuts lie.
struct Cuts {
  int k;     // the k-th token's bin, or -1
  int2 p, u;  // where top-p's and the drawn token may be, from bounds on the masses before them
  int first, last;
  uint64_t all, from_min;

  __device__ __forceinline__ bool has(int b) const {
    if (b < first || b > last) return false;  // as most
    return b == k || (b >= p.x && b <= p.y) || (b >= u.x && b <= u.y);
  }
};

// From the histogram's exclusive counts (with top-k, whose bin is bk) and its masses.
__device__ __forceinline__ Cuts cuts_of(Shared& sh, const Settings& st, int bk) {
  const Span own = scan_bins<kBins, true, false>(sh, sh.mass, sh.count, 0, 0);
  Cuts c;
  c.all = sh.all, c.from_min = st.by_min ? sh.least : c.all;
  c.k = bk;
  c.p = make_int2(-1, -2);
  const double u = st.number(), share = st.share();
  auto at = [&](int b) { return sh.mass[place<kBins>(b)]; };
  auto after = [&](int b) { return b + 1 < kBins ? at(b + 1) : c.all; };
  uint64_t lo = c.all, hi = c.all;
  if (bk >= 0) lo = at(bk), hi = after(bk);
  if (st.by_p) {
    c.p = bins_of<kReach, kBins>(sh, sh.mass, sh.count, own, share * static_cast<double>(lo), share * static_cast<double>(hi));
    lo = min(lo, at(c.p.x)), hi = min(hi, after(c.p.y));
  }
  lo = min(lo, c.from_min), hi = min(hi, c.from_min);
  c.u = bins_of<kPass, kBins>(sh, sh.mass, sh.count, own, u * static_cast<double>(lo), u * static_cast<double>(hi));
  c.first = st.by_p ? min(c.p.x, c.u.x) : c.u.x, c.last = max(max(c.k, c.p.y), c.u.y);
  return c;
}

// The tokens of the cuts' bins, put(slot, token) in any order; counts them all.
template <typename Put>
__device__ __forceinline__ void gather(const Scale& sc, const Cuts& c, Logits& l, uint32_t* n_list, Put put) {
  l.every([&](float x, int i) {
    const int b = sc.bin(x);
    if (!c.has(b)) return;
    const uint64_t w = sc.weight(x);
    if (!w) return;
    const uint32_t slot = atomicAdd(n_list, 1u);
    if (slot < kList)
      put(slot, Token{static_cast<uint64_t>(order_key(x)) << 32 | static_cast<uint32_t>(b) << 19 | (kMostTokens - i), w}, b);
  });
}

// The choice among the m gathered tokens of sh.list; earlier(slot, mass, count): of the bins
// before a token's.
template <typename Earlier>
__device__ __forceinline__ void choose(Shared& sh, const SampleArgs& a, const Settings& st, const Scale& sc, int t, int m, uint64_t all,
                       uint64_t from_min, bool infinite, float low, Earlier earlier) {
  const int tid = threadIdx.x;
  const double u = st.number(), share = st.share();
  uint64_t M = all;
  End end;
  if (m <= kList) {
    // P threads to a token, each of which looks at every P-th of the others
    int P = 64;
    while (P > 1 && P * m > kThreads) P /= 2;
    const int e = tid / P;
    uint64_t before = 0, own = 0, order = 0;
    uint32_t rank = 0;
    if (e < m) {
      order = sh.list[e].order, own = sh.list[e].weight;
      for (int j = tid % P; j < m; j += P) {
        const Token x = sh.list[j];
        if (x.order > order && !(static_cast<uint32_t>(x.order ^ order) >> 19)) before += x.weight, ++rank;
      }
    }
    for (int s = P / 2; s >= 1; s >>= 1) {
      before += __shfl_xor(static_cast<unsigned long long>(before), s, 64);
      rank += __shfl_xor(rank, s, 64);
    }
    if (e < m) earlier(e, static_cast<uint32_t>(order) >> 19, before, rank);
    const int token = kMostTokens - static_cast<int>(order & kMostTokens);
    if (st.by_k) M = min(M, cut_in_list<kCount>(sh, st.k, before, rank, own, token).mass);
    if (st.by_p) M = min(M, cut_in_list<kReach>(sh, share * static_cast<double>(M), before, rank, own, token).mass);
    M = min(M, from_min);
    end = cut_in_list<kPass>(sh, u * static_cast<double>(M), before, rank, own, token);
  } else {
    const float* row = a.logits + static_cast<size_t>(t) * a.n;
    if (st.by_k) M = min(M, cut_in_row<kCount>(sh, sc, row, a.n, infinite, low, st.k).mass);
    if (st.by_p) M = min(M, cut_in_row<kReach>(sh, sc, row, a.n, infinite, low, share * static_cast<double>(M)).mass);
    M = min(M, from_min);
    end = cut_in_row<kPass>(sh, sc, row, a.n, infinite, low, u * static_cast<double>(M));
  }
  if (tid == 0) {
    a.idx[t] = end.token;
    if (a.prob) a.prob[t] = static_cast<float>(static_cast<double>(end.weight) / static_cast<double>(M));
  }
}

// A work-group per row.  What costs most is the weights, in double precision: with top-k, or
// min-p alone, only the tokens down to a cut's bin are weighed.
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int t = blockIdx.x, tid = threadIdx.x;
  Logits l(a.logits + static_cast<size_t>(t) * a.n, 0, a.n);
  const Settings st(a, t);
  tabulate(sh);
  clear(sh);
  if (tid == 0) sh.n_list = 0, sh.found_at = a.n;
  float2 r = range_of(sh, l);
  if (st.greedy(r.x)) {
    int at = a.n;
    l.every([&](float x, int i) { at = x == r.x && i < at ? i : at; });
    if (at < a.n) atomicMin(&sh.found_at, at);
    __syncthreads();
    if (tid == 0) {
      a.idx[t] = r.x > -INFINITY ? sh.found_at : 0;
      if (a.prob) a.prob[t] = 1.0f;
    }
    return;
  }
  if (r.x == INFINITY) l.make_infinite(), r = make_float2(0.0f, -INFINITY);
  const Scale sc = st.scale(sh, r.x, r.y);
  int last = kBins - 1;  // the last bin that matters
  if (st.by_min && !st.by_p)  // (a bin further, for its fp32 distances)
    last = static_cast<int>(fminf(-logf(fminf(st.min_p, 1.0f)) * st.temp * 1.00001f * sc.bins, kBins - 2)) + 1;
  if (st.by_k) {
    l.every([&](float x, int) { count_token(sh, sc.bin(x)); });
    __syncthreads();
    const Span own = scan_bins<kBins, false, true>(sh, sh.mass, sh.count, 0, 0);
    last = min(last, bins_of<kCount, kBins>(sh, sh.mass, sh.count, own, st.k, st.k).x);
  }
  weigh<false>(sh, sc, st, l, last);
  __syncthreads();
  const Cuts c = cuts_of(sh, st, st.by_k ? last : -1);  // (a bin before the k-th token's where min_p ends there)
  gather(sc, c, l, &sh.n_list, [&](uint32_t slot, Token x, int) { sh.list[slot] = x; });
  __syncthreads();
  choose(sh, a, st, sc, t, static_cast<int>(sh.n_list), c.all, c.from_min, l.infinite, r.y,
         [&](int, uint32_t b, uint64_t& mass, uint32_t& count) { mass += sh.mass[place<kBins>(b)], count += sh.count[place<kBins>(b)]; });
}

// The same by several work-groups a row, in four launches: the range of each, one histogram of
// them all, the tokens of the cuts' bins, and the choice.
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
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64)), low = fminf(low, __shfl_xor(low, s, 64));
    return make_float2(top, low);
  }
};
__device__ __forceinline__ SplitRow& split_row(const SampleArgs& a, int t) { return static_cast<SplitRow*>(a.workspace)[t]; }
__device__ __forceinline__ Logits share_of(const SampleArgs& a, int s, int t) {
  return Logits(a.logits + static_cast<size_t>(t) * a.n, min(s * a.share, a.n), min((s + 1) * a.share, a.n));
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

__global__ __launch_bounds__(kThreads) void sample_range_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const auto [s, t] = part_of(a);
  if (t >= a.T) return;
  SplitRow& ws = split_row(a, t);
  Logits l = share_of(a, s, t);
  for (int b = s * kThreads + static_cast<int>(threadIdx.x); b < kBins; b += a.splits * kThreads) ws.mass[b] = 0, ws.count[b] = 0;
  if (s == 0 && threadIdx.x == 0) ws.least = 0, ws.n_list = 0, ws.at = a.n;
  const float2 r = range_of(sh, l);
  if (threadIdx.x == 0) ws.range[s] = r;
}

__global__ __launch_bounds__(kThreads) void sample_weigh_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const auto [s, t] = part_of(a);
  const int tid = threadIdx.x;
  if (t >= a.T) return;
  SplitRow& ws = split_row(a, t);
  Logits l = share_of(a, s, t);
  const Settings st(a, t);
  tabulate(sh);
  clear(sh);
  float2 r = ws.whole(a.splits);
  if (st.greedy(r.x)) {
    int at = a.n;
    l.every([&](float x, int i) { at = x == r.x && i < at ? i : at; });
    if (at < a.n && r.x > -INFINITY) atomicMin(&ws.at, at);
    return;
  }
  if (r.x == INFINITY) l.make_infinite(), r = make_float2(0.0f, -INFINITY);
  const Scale sc = st.scale(sh, r.x, r.y);
  __syncthreads();
  weigh<true>(sh, sc, st, l, kBins - 1);
  __syncthreads();
#pragma unroll
  for (int b = 0; b < kBins; b += kThreads) {
    if (const uint64_t x = sh.mass[b + tid]) atomicAdd(reinterpret_cast<unsigned long long*>(ws.mass + b + tid), x);
    if (const uint32_t x = sh.count[b + tid]) atomicAdd(ws.count + b + tid, x);
  }
  if (tid == 0 && sh.least) atomicAdd(reinterpret_cast<unsigned long long*>(&ws.least), sh.least);
}

__global__ __launch_bounds__(kThreads) void sample_gather_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const auto [s, t] = part_of(a);
  const int tid = threadIdx.x;
  if (t >= a.T) return;
  SplitRow& ws = split_row(a, t);
  Logits l = share_of(a, s, t);
  const Settings st(a, t);
#pragma unroll
  for (int b = 0; b < kBins; b += kThreads) sh.mass[b + tid] = ws.mass[b + tid], sh.count[b + tid] = ws.count[b + tid];
  if (tid == 0) sh.least = ws.least;
  tabulate(sh);
  float2 r = ws.whole(a.splits);
  if (st.greedy(r.x)) return;
  if (r.x == INFINITY) l.make_infinite(), r = make_float2(0.0f, -INFINITY);
  const Scale sc = st.scale(sh, r.x, r.y);
  __syncthreads();
  int bk = -1;
  if (st.by_k) {
    const Span own = scan_bins<kBins, false, true>(sh, sh.mass, sh.count, 0, 0);
    bk = bins_of<kCount, kBins>(sh, sh.mass, sh.count, own, st.k, st.k).x;
  }
  const Cuts c = cuts_of(sh, st, bk);
  gather(sc, c, l, &ws.n_list, [&](uint32_t slot, Token x, int b) {
    ws.list[slot] = {x, sh.mass[place<kBins>(b)], sh.count[place<kBins>(b)]};
  });
  if (s == 0 && tid == 0) ws.all = c.all;
}

__global__ __launch_bounds__(kThreads) void sample_choose_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int t = blockIdx.x, tid = threadIdx.x;
  const SplitRow& ws = split_row(a, t);
  const Settings st(a, t);
  tabulate(sh);
  float2 r = ws.whole(a.splits);
  if (st.greedy(r.x)) {
    if (tid == 0) {
      a.idx[t] = r.x > -INFINITY ? ws.at : 0;
      if (a.prob) a.prob[t] = 1.0f;
    }
    return;
  }
  const bool infinite = r.x == INFINITY;
  if (infinite) r = make_float2(0.0f, -INFINITY);
  const int m = static_cast<int>(ws.n_list);
  if (m <= kList && tid < m) sh.list[tid] = ws.list[tid].token;
  __syncthreads();
  choose(sh, a, st, st.scale(sh, r.x, r.y), t, m, ws.all, st.by_min ? ws.least : ws.all, infinite, r.y,
         [&](int e, uint32_t, uint64_t& mass, uint32_t& count) { mass += ws.list[e].mass, count += static_cast<uint32_t>(ws.list[e].count); });
}

// Work-groups of a row: one where it holds the row in registers, else as many as leave one a
// CU of the XCD that the row's are on, of at least kLeastShare logits each.  One | several, us:
// one row of 50257 47 | 28, of 131071 73 | 29; 64 rows of 131071 95 | 53; 128 rows of 131071 100 | 86;
// but of 32000 one row 18 | 29, 64 rows 19 | 44, 128 rows 19 | 50.
constexpr int kLeastShare = 4096;
int splits_of(int T, int n) {
  const int rows = (std::max(T, 1) - 1) / kXcds + 1;  // of an XCD
  return n <= kHold * kThreads ? 1 : std::max(1, std::min(kCus / kXcds / rows, n / kLeastShare));
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
  if (T > UINT32_MAX / kThreads) return MS_E_UNSUPPORTED;
  const int splits = splits_of(T, n);
  SampleArgs a = {logits, u_dev, nullptr, nullptr, nullptr, nullptr, idx_out, prob_out, T, n, splits, (n - 1) / splits + 1, workspace_dev};
  if (opts) a.temperature = opts->temperature_dev, a.top_p = opts->top_p_dev, a.min_p = opts->min_p_dev, a.top_k = opts->top_k_dev;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 rows(static_cast<unsigned>(T)), all((static_cast<unsigned>(T) + kXcds - 1) / kXcds * kXcds * splits), block(kThreads);
  if (splits == 1) {
    hipLaunchKernelGGL(sample_kernel, rows, block, 0, s, a);
  } else {
    hipLaunchKernelGGL(sample_range_kernel, all, block, 0, s, a);
    hipLaunchKernelGGL(sample_weigh_kernel, all, block, 0, s, a);
    hipLaunchKernelGGL(sample_gather_kernel, all, block, 0, s, a);
    hipLaunchKernelGGL(sample_choose_kernel, rows, block, 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP;
}

}  // extern "C"
