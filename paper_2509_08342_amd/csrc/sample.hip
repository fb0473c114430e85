// A token drawn from each row of logits: temperature, top-k, top-p and min-p, from given
// random numbers.  Stateless, like the other calls of the decoder loop.
//
// With the logits l in descending order, ties to the lower index, and weights
// exp((l - max) / temperature), every filter keeps a prefix, so the kept mass M is the least
// of the filters' masses, and the token is the first whose running mass passes u M.  No row
// is sorted: a histogram over the distance from the maximum gives the running mass at 2048
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
constexpr double kFar = 31.9;    // exp(-kFar) rounds to zero units

__device__ __forceinline__ float logit(float x) { return x == x ? x : -INFINITY; }

// order of fp32 values as unsigned numbers; -0 and 0 alike
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// What a row's tokens are weighed with.
struct Scale {
  double inv;  // 1 / temperature
  float top;   // the largest logit
  float bins;  // per unit of distance
  const double* powers;  // 2^(-i / 64)

  // (top - l) / temperature, 0 at the maximum even if that is infinite
  __device__ __forceinline__ double away(float l) const { return l == top ? 0.0 : (static_cast<double>(top) - l) * inv; }
  __device__ __forceinline__ int bin(double d) const { return static_cast<int>(fminf(static_cast<float>(d) * bins, kBins - 1)); }
  // exp(-d) in units: 2^(-j / 64) from the table and the series of the rest, |r| <= ln 2 / 128,
  // to r^5 / 120 (the next term is 2^-54)
  __device__ __forceinline__ uint64_t weight(double d) const {
    if (!(d < kFar)) return 0;
    const double j = rint(d * 92.332482616893656877);  // 64 / ln 2
    const double r = fma(j, -0.010830424696249145251, d);  // ln 2 / 64
    double s = fma(r, -1.0 / 120, 1.0 / 24);
    s = fma(r, s, -1.0 / 6);
    s = fma(r, s, 0.5);
    s = fma(r, s, -1.0);
    s = fma(r, s, 1.0);
    const int i = static_cast<int>(j);
    const double e = s * powers[i & 63];
    const long long scaled = __double_as_longlong(e) + (static_cast<long long>(45 - (i >> 6)) << 52);
    // rounds to a whole number in the low bits
    return static_cast<uint64_t>(__double_as_longlong(__longlong_as_double(scaled) + 4503599627370496.0)) & ((1ull << 52) - 1);
  }
};

struct SampleArgs {
  const float *logits, *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* idx;
  float* prob;
  int n;
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
  double powers[64];
  uint64_t wave_mass[kThreads / 64];
  uint32_t wave_count[kThreads / 64];
  float wave_top[kThreads / 64], wave_low[kThreads / 64];
  int32_t wave_at[kThreads / 64];
  uint64_t all, least, found_mass, found_weight;
  uint32_t all_count, n_list;
  int32_t found_at;
};

// Exclusive sums of mass and count in place; the totals to sh.all and sh.all_count.
template <int BINS>
__device__ void scan_bins(Shared& sh, uint64_t* mass, uint32_t* count, uint64_t mass0, uint32_t count0) {
  constexpr int PER = BINS / kThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t m = 0;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) m += mass[tid * PER + i], c += count[tid * PER + i];
  uint64_t im = m;
  uint32_t ic = c;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint64_t om = __shfl_up(static_cast<unsigned long long>(im), s, 64);
    const uint32_t oc = __shfl_up(ic, s, 64);
    if (lane >= s) im += om, ic += oc;
  }
  if (lane == 63) sh.wave_mass[wave] = im, sh.wave_count[wave] = ic;
  __syncthreads();
  uint64_t base = mass0 + im - m;
  uint32_t bc = count0 + ic - c;
  for (int w = 0; w < wave; ++w) base += sh.wave_mass[w], bc += sh.wave_count[w];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t x = mass[tid * PER + i];
    const uint32_t y = count[tid * PER + i];
    mass[tid * PER + i] = base, count[tid * PER + i] = bc;
    base += x, bc += y;
  }
  if (tid == kThreads - 1) sh.all = base, sh.all_count = bc;
  __syncthreads();
}

// Where a prefix ends: at the token that makes it t long, that takes its mass to t, or past t.
enum Cut { kCount, kReach, kPass };

// Whether the prefix before `mass` and `count` is still short of the cut.
template <Cut CUT>
__device__ __forceinline__ bool is_short(double t, uint64_t mass, uint32_t count) {
  return CUT == kCount ? count < t : CUT == kReach ? static_cast<double>(mass) < t : static_cast<double>(mass) <= t;
}

// The bin in which the cut lies, from exclusive sums.
template <Cut CUT>
__device__ __forceinline__ int bin_of(const uint64_t* mass, const uint32_t* count, int bins, double t) {
  int lo = 0, hi = bins - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (is_short<CUT>(t, mass[mid], count[mid]))
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

struct End {
  uint64_t mass, weight;  // of the prefix, the token at its end included, and of that token
  int token;
};

// A cut among the gathered tokens: each knows what is before it, and one of them is the end.
template <Cut CUT>
__device__ End cut_in_list(Shared& sh, double t, int m, uint64_t before, uint32_t rank, uint64_t own, int token) {
  if (static_cast<int>(threadIdx.x) < m && !is_short<CUT>(t, before + own, rank + 1) &&
      (is_short<CUT>(t, before, rank) || before == 0))
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
__device__ End cut_in_row(Shared& sh, const Scale& sc, const float* row, int n, float low, double t) {
  const int tid = threadIdx.x;
  uint32_t kmax = order_key(sc.top), kmin = order_key(low);
  uint64_t base = 0;
  uint32_t rank = 0;
  while (kmax > kmin) {
    const int shift = max(0, 32 - __clz(kmax - kmin) - 10);
    sh.sub.mass[tid] = 0, sh.sub.count[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const float l = logit(row[i]);
      const uint32_t key = order_key(l);
      if (!(l > -INFINITY) || key < kmin || key > kmax) continue;
      const uint64_t w = sc.weight(sc.away(l));
      if (!w) continue;
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.sub.mass[(kmax - key) >> shift]), w);
      atomicAdd(&sh.sub.count[(kmax - key) >> shift], 1u);
    }
    __syncthreads();
    scan_bins<kSubBins>(sh, sh.sub.mass, sh.sub.count, base, rank);
    const uint32_t b = bin_of<CUT>(sh.sub.mass, sh.sub.count, kSubBins, t);
    base = sh.sub.mass[b], rank = sh.sub.count[b];
    kmax -= b << shift;
    kmin = max(kmin, kmax - ((1u << shift) - 1));
    __syncthreads();
  }
  // the tokens of one value, by their index: the first with enough before it
  const uint64_t w = sc.weight(sc.away(key_value(kmax)));
  if (tid == 0) sh.found_at = -1;
  __syncthreads();
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + tid;
    const bool is = i < n && order_key(logit(row[i])) == kmax;
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

__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n;
  const float* row = a.logits + static_cast<size_t>(t) * n;
  if (tid < 64) sh.powers[tid] = exp2(-tid / 64.0);
  for (int b = tid; b < kBins; b += kThreads) sh.mass[b] = 0, sh.count[b] = 0;
  if (tid == 0) sh.n_list = 0, sh.least = 0;

  // the largest logit, its first place, and the smallest above -infinity
  float top = -INFINITY, low = INFINITY;
  int at = n;
  for (int i = tid; i < n; i += kThreads) {
    const float l = logit(row[i]);
    if (l > top) top = l, at = i;
    if (l > -INFINITY) low = fminf(low, l);
  }
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) {
    const float ot = __shfl_xor(top, s, 64);
    const int oa = __shfl_xor(at, s, 64);
    if (ot > top || (ot == top && oa < at)) top = ot, at = oa;
    low = fminf(low, __shfl_xor(low, s, 64));
  }
  if (lane == 0) sh.wave_top[wave] = top, sh.wave_low[wave] = low, sh.wave_at[wave] = at;
  __syncthreads();
  for (int w = 0; w < kThreads / 64; ++w) {
    const float ot = sh.wave_top[w];
    const int oa = sh.wave_at[w];
    if (ot > top || (ot == top && oa < at)) top = ot, at = oa;
    low = fminf(low, sh.wave_low[w]);
  }
  const float temp = a.temperature ? a.temperature[t] : 1.0f;
  if (!(temp > 0.0f) || top == -INFINITY) {  // the arg max
    if (tid == 0) {
      a.idx[t] = at < n ? at : 0;
      if (a.prob) a.prob[t] = 1.0f;
    }
    return;
  }
  Scale sc;
  sc.inv = 1.0 / temp;
  sc.top = top;
  sc.powers = sh.powers;
  const float span = static_cast<float>(fmin(sc.away(low), kFar));
  sc.bins = span > 0.0f ? (kBins - 1) / span : 0.0f;
  const int k = a.top_k ? a.top_k[t] : 0;
  const float p = a.top_p ? a.top_p[t] : 1.0f, min_p = a.min_p ? a.min_p[t] : 0.0f;
  const bool by_k = k > 0 && k < n, by_p = p < 1.0f, by_min = min_p > 0.0f;
  const double least = fmin(static_cast<double>(min_p), 1.0) * kUnit;

  uint64_t kept = 0;  // of tokens that min_p keeps
  for (int i = tid; i < n; i += kThreads) {
    const float l = logit(row[i]);
    const double d = sc.away(l);
    const uint64_t w = l > -INFINITY ? sc.weight(d) : 0;
    if (w) {
      const int b = sc.bin(d);
      atomicAdd(reinterpret_cast<unsigned long long*>(&sh.mass[b]), w);
      if (by_k) atomicAdd(&sh.count[b], 1u);
      if (static_cast<double>(w) >= least) kept += w;
    }
  }
  if (by_min) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.least), kept);
  __syncthreads();
  scan_bins<kBins>(sh, sh.mass, sh.count, 0, 0);

  const double u = fmin(fmax(a.u[t], 0.0f), 0x1.fffffep-1f);  // a NaN draws as 0
  const double share = fmax(static_cast<double>(p), 0.0);
  const uint64_t all = sh.all, from_min = by_min ? sh.least : all;
  const bool cut_k = by_k && static_cast<uint32_t>(k) < sh.all_count;
  auto bin = [&](auto cut, double x) { return bin_of<decltype(cut)::value>(sh.mass, sh.count, kBins, x); };
  using Count = std::integral_constant<Cut, kCount>;
  using Reach = std::integral_constant<Cut, kReach>;
  using Pass = std::integral_constant<Cut, kPass>;
  auto after = [&](int b) { return b + 1 < kBins ? sh.mass[b + 1] : all; };
  // the bins in which the cuts lie, from bounds on the masses that they leave
  uint64_t lo = all, hi = all;
  int bk = -1, bp0 = -1, bp1 = -2;
  if (cut_k) {
    bk = bin(Count{}, k);
    lo = sh.mass[bk], hi = after(bk);
  }
  if (by_p) {
    bp0 = bin(Reach{}, share * static_cast<double>(lo)), bp1 = bin(Reach{}, share * static_cast<double>(hi));
    lo = min(lo, sh.mass[bp0]), hi = min(hi, after(bp1));
  }
  lo = min(lo, from_min), hi = min(hi, from_min);
  const int bu0 = bin(Pass{}, u * static_cast<double>(lo)), bu1 = bin(Pass{}, u * static_cast<double>(hi));
  for (int i = tid; i < n; i += kThreads) {
    const float l = logit(row[i]);
    const double d = sc.away(l);
    if (!(l > -INFINITY) || !(d < kFar)) continue;
    const int b = sc.bin(d);
    if (b != bk && !(b >= bp0 && b <= bp1) && !(b >= bu0 && b <= bu1)) continue;
    const uint64_t w = sc.weight(d);
    if (!w) continue;
    const uint32_t slot = atomicAdd(&sh.n_list, 1u);
    if (slot < kList)
      sh.list[slot] = {static_cast<uint64_t>(order_key(l)) << 32 | static_cast<uint32_t>(b) << 19 | (kMostTokens - i), w};
  }
  __syncthreads();
  const int m = static_cast<int>(sh.n_list);
  uint64_t M = all;
  End end;
  if (m <= kList) {
    uint64_t before = 0, own = 0, order = 0;
    uint32_t rank = 0;
    if (tid < m) {
      order = sh.list[tid].order, own = sh.list[tid].weight;
      const int b = static_cast<uint32_t>(order) >> 19;
      before = sh.mass[b], rank = sh.count[b];
      for (int j = 0; j < m; ++j) {
        const Token x = sh.list[j];
        if (x.order > order && !(static_cast<uint32_t>(x.order ^ order) >> 19)) before += x.weight, ++rank;
      }
    }
    const int token = kMostTokens - static_cast<int>(order & kMostTokens);
    if (cut_k) M = cut_in_list<kCount>(sh, k, m, before, rank, own, token).mass;
    if (by_p) M = min(M, cut_in_list<kReach>(sh, share * static_cast<double>(M), m, before, rank, own, token).mass);
    M = min(M, from_min);
    end = cut_in_list<kPass>(sh, u * static_cast<double>(M), m, before, rank, own, token);
  } else {
    if (cut_k) M = cut_in_row<kCount>(sh, sc, row, n, low, k).mass;
    if (by_p) M = min(M, cut_in_row<kReach>(sh, sc, row, n, low, share * static_cast<double>(M)).mass);
    M = min(M, from_min);
    end = cut_in_row<kPass>(sh, sc, row, n, low, u * static_cast<double>(M));
  }
  if (tid == 0) {
    a.idx[t] = end.token;
    if (a.prob) a.prob[t] = static_cast<float>(static_cast<double>(end.weight) / static_cast<double>(M));
  }
}

}  // namespace

extern "C" {

ms_status ms_sample_workspace(int32_t T, int32_t n, uint64_t* bytes_out) {
  if (T < 0 || n <= 0 || !bytes_out) return MS_E_INVALID;
  if (n > kMostTokens) return MS_E_UNSUPPORTED;
  *bytes_out = 0;
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
  SampleArgs a = {logits, u_dev, nullptr, nullptr, nullptr, nullptr, idx_out, prob_out, n};
  if (opts) a.temperature = opts->temperature_dev, a.top_p = opts->top_p_dev, a.min_p = opts->min_p_dev, a.top_k = opts->top_k_dev;
  hipLaunchKernelGGL(sample_kernel, dim3(static_cast<unsigned>(T)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? MS_OK : MS_E_HIP;
}

}  // extern "C"
