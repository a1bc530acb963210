// Sampling from the target's logits with given random numbers.
//
// Row of logits l, temperature T: weights w_i = e^((l_i - max) / T).  What is kept
// is cut down in turn: weights of at least min_p (times the largest, 1), then the
// top_k largest, then the smallest set of largest weights that reaches top_p of
// their sum; equal logits count in vocabulary order.  The token is the first of
// the kept ones, in vocabulary order, whose running sum of weights passes
// uniform * total.
//
// A token is a whole number, and there are up to V borders between tokens: with
// sums in 32 bits (1e-7 off) a row of 150,000 open tokens would now and then get
// its neighbour.  Weights and sums are float64, which this card computes at the
// rate of float32; the histograms' sums are whole numbers, so that the order of
// their atomics does not matter.
//
// Two launches.  scan_kernel reads the logits once: maxima of groups of 64
// logits, and for the rows that need all of it (no top_k, no min_p) the sum of
// weights of each block of 512.  pick_kernel, one workgroup a row, starts from
// those.  With a top_k of at most the number of groups, the k-th largest group
// maximum is a lower bound of the k-th largest logit, so only groups that reach
// it are read again, and what reaches it, hardly more than k logits, is sorted in
// LDS; min_p gives such a bound too, and a top_p alone first tries the logits
// from the 256-th largest group maximum up.  Rows that this does not settle are
// cut by histograms over the whole row.
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pctree_sample.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr int kUnit = 8;              // consecutive logits of a lane
constexpr int kBlock = 64 * kUnit;    // logits of a wave's step
constexpr int kMaxGroups = 2561;      // of a row
constexpr int kMaxBlocks = PCTREE_MAX_VOCAB / kBlock + 1;
constexpr int kScanThreads = 256;
constexpr int kPickThreads = 512;
constexpr int kPickWaves = kPickThreads / 64;
constexpr int kList = 2048;           // logits sorted in LDS
constexpr int kBins = 2048;
constexpr double kLowest = -700.0;    // weights below e^-700 are 0
constexpr double kLog2e = 1.4426950408889634074;

// 2^r, |r| <= 1/2, by its Taylor series (the thirteenth term is below 2^-53).
__device__ __forceinline__ double exp2_small(double r) {
  constexpr double L = 0.69314718055994530942;
  constexpr double c1 = L, c2 = c1 * L / 2, c3 = c2 * L / 3, c4 = c3 * L / 4, c5 = c4 * L / 5,
                   c6 = c5 * L / 6, c7 = c6 * L / 7, c8 = c7 * L / 8, c9 = c8 * L / 9,
                   c10 = c9 * L / 10, c11 = c10 * L / 11, c12 = c11 * L / 12;
  double s = c12;
  s = __builtin_fma(s, r, c11);
  s = __builtin_fma(s, r, c10);
  s = __builtin_fma(s, r, c9);
  s = __builtin_fma(s, r, c8);
  s = __builtin_fma(s, r, c7);
  s = __builtin_fma(s, r, c6);
  s = __builtin_fma(s, r, c5);
  s = __builtin_fma(s, r, c4);
  s = __builtin_fma(s, r, c3);
  s = __builtin_fma(s, r, c2);
  s = __builtin_fma(s, r, c1);
  return __builtin_fma(s, r, 1.0);
}
// e^z for z in [-700, 0]; 0 below (and for NaN).
__device__ __forceinline__ double weight_of(double z) {
  const double t = z * kLog2e, n = __builtin_rint(t);
  const double w = __builtin_ldexp(exp2_small(t - n), (int)n);
  return z >= kLowest ? w : 0.0;
}

// Floats as whole numbers of the same order (-0 as +0), and back.
__device__ __forceinline__ uint32_t ord_of(float v) {
  const uint32_t b = __float_as_uint(v == 0.0f ? 0.0f : v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_ord(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// A row at any alignment: `base` is its start rounded down to 16 bytes, and logit
// i is element lo + i from there, i < V.  Units of 8 elements from base on are a
// lane's share; NaN counts as -inf, and so does what lies outside the row.
struct Row {
  const char* base;
  int lo, hi;
};
template <int DT>
__device__ __forceinline__ Row row_of(const SampleArgs& a, int t) {
  constexpr int ES = DT == PCTREE_F32 ? 4 : 2;
  const char* p = (const char*)a.logits + (long long)t * a.row_stride * ES;
  Row r;
  r.base = (const char*)((uintptr_t)p & ~(uintptr_t)15);
  r.lo = (int)((p - r.base) / ES);
  r.hi = r.lo + a.V;
  return r;
}
template <int DT>
__device__ __forceinline__ void load_unit(const Row& r, int u, float (&v)[kUnit]) {
  const int j0 = u * kUnit;
  if (j0 >= r.lo && j0 + kUnit <= r.hi) {
    if constexpr (DT == PCTREE_F32) {
      const f32x4* p = (const f32x4*)(r.base + (size_t)j0 * 4);
      const f32x4 x = p[0], y = p[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = x[e];
        v[4 + e] = y[e];
      }
    } else {
      const u32x4 x = *(const u32x4*)(r.base + (size_t)j0 * 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = lo16<DT == PCTREE_F16>(x[e]);
        v[2 * e + 1] = hi16<DT == PCTREE_F16>(x[e]);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      v[e] = kNegInf;
      if (j0 + e >= r.lo && j0 + e < r.hi) {
        if constexpr (DT == PCTREE_F32)
          v[e] = ((const float*)r.base)[j0 + e];
        else
          v[e] = lo16<DT == PCTREE_F16>(((const uint16_t*)r.base)[j0 + e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kUnit; ++e) v[e] = v[e] == v[e] ? v[e] : kNegInf;
}

// A row's parameters.
struct Params {
  double inv_t, p, min_p, u;
  int k;        // 0: off
  bool greedy;  // a temperature of 0 (or below, or NaN): the largest logit
};
__device__ __forceinline__ Params params_of(const SampleArgs& a, int t) {
  Params q;
  const float T = a.temperature ? a.temperature[t] : 1.0f;
  q.greedy = !(T > 0.0f);
  q.inv_t = q.greedy ? 1.0 : 1.0 / (double)T;
  const int k = a.top_k ? a.top_k[t] : 0;
  q.k = k > 0 && k < a.V ? k : 0;
  const float p = a.top_p ? a.top_p[t] : 1.0f;
  q.p = p < 1.0f ? (double)p : 1.0;  // (NaN: off)
  const float m = a.min_p ? a.min_p[t] : 0.0f;
  q.min_p = m > 0.0f ? (double)fminf(m, 1.0f) : 0.0;
  const float u = a.uniform[t];
  q.u = u > 0.0f ? (double)u : 0.0;
  return q;
}
// Whether the row is settled from its largest logits, without the sum of all.
__device__ __forceinline__ bool bounded(const SampleArgs& a, const Params& q) {
  return q.greedy || q.min_p > 0.0 || (q.k > 0 && q.k <= a.ng);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

template <int DT, int BPW>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(SampleArgs a, int segs) {
  const int t = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int lane = threadIdx.x & 63;
  const int b0 = (seg * (kScanThreads / 64) + threadIdx.x / 64) * BPW;
  if (b0 >= a.nb) return;
  const Row row = row_of<DT>(a, t);
  float v[BPW][kUnit], mx[BPW];
#pragma unroll
  for (int i = 0; i < BPW; ++i) load_unit<DT>(row, (b0 + i) * 64 + lane, v[i]);
  const int lanes = 8 << a.gshift;  // of a group
  float all = kNegInf;
#pragma unroll
  for (int i = 0; i < BPW; ++i) {
    mx[i] = v[i][0];
#pragma unroll
    for (int e = 1; e < kUnit; ++e) mx[i] = fmaxf(mx[i], v[i][e]);
    all = fmaxf(all, mx[i]);
    for (int o = 1; o < lanes; o <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor(mx[i], o, 64));
    const int g = ((b0 + i) * 64 + lane) / lanes;
    if (lane % lanes == 0 && g < a.ng) a.gmax[(size_t)t * a.ng + g] = mx[i];
  }
  const Params q = params_of(a, t);
  if (bounded(a, q)) return;
  const float ref = wave_max(all);
#pragma unroll
  for (int i = 0; i < BPW; ++i) {
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < kUnit; ++e)
      s += v[i][e] == ref ? 1.0 : weight_of(((double)v[i][e] - (double)ref) * q.inv_t);
    s = wave_sum(s);
    if (lane == 0 && b0 + i < a.nb) {
      a.bmass[(size_t)t * a.nb + b0 + i] = ref == kNegInf ? 0.0 : s;
      a.bref[(size_t)t * a.nb + b0 + i] = ref;
    }
  }
}

// ---------------------------------------------------------------------------
// pick: one workgroup a row
// ---------------------------------------------------------------------------

struct PickShared {
  float gmax[kMaxGroups + 3];
  union {
    struct {
      uint64_t list[kList];
      double w[kList];
    } l;
    struct {
      unsigned long long mass[kBins];
      uint32_t count[kBins];
    } h;
    struct {
      double mass[kMaxBlocks + 1];
      int ties[kMaxBlocks + 1];
    } b;
  };
  double part[kPickWaves];
  int parti[kPickWaves];
  int n, found, extra;
  uint32_t lo, hi;
};

__device__ __forceinline__ double block_sum(double v, PickShared& sh) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w) s += sh.part[w];
  return s;
}
__device__ __forceinline__ int block_sum(int v, PickShared& sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.parti[threadIdx.x >> 6] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w) s += sh.parti[w];
  return s;
}
// Sum over the threads before this one (always added in the same order).
__device__ __forceinline__ double block_before(double v, PickShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) sh.part[wave] = x;
  __syncthreads();
  double b = __shfl_up(x, 1, 64);
  if (lane == 0) b = 0.0;
  double base = 0.0;
  for (int w = 0; w < wave; ++w) base += sh.part[w];
  return base + b;
}
__device__ __forceinline__ int block_before(int v, PickShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) sh.parti[wave] = x;
  __syncthreads();
  int base = x - v;
  for (int w = 0; w < wave; ++w) base += sh.parti[w];
  return base;
}

// The j-th largest group maximum (j >= 1; all of them: -inf), as a float whose
// low 12 bits may be rounded down.
__device__ float group_bound(const SampleArgs& a, int j, PickShared& sh) {
  uint32_t lo = 0;  // at least j maxima are >= lo
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t mid = lo | (1u << bit);
    int c = 0;
    for (int g = threadIdx.x; g < a.ng; g += kPickThreads) c += ord_of(sh.gmax[g]) >= mid;
    if (block_sum(c, sh) >= j) lo = mid;
  }
  return lo < 0x00800000u ? kNegInf : of_ord(lo);
}

// Logits >= bound into the list (unordered), as (order, lowest index first);
// returns how many there are (more than kList: not all are in the list).
template <int DT>
__device__ int gather(const SampleArgs& a, const Row& row, float bound, PickShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  const int per = 8 << a.gshift;  // units of a group
  // a wave takes 64 / 8 groups of 64 logits at a time
  const int step = 64 / per;
  for (int g0 = wave * step; g0 < a.ng; g0 += kPickWaves * step) {
    const int g = g0 + lane / per;
    const bool in = g < a.ng && sh.gmax[min(g, a.ng - 1)] >= bound;
    if (!__any(in)) continue;
    float v[kUnit];
    const int u = g * per + lane % per;
    int hits = 0;
    if (in) {
      load_unit<DT>(row, u, v);
#pragma unroll
      for (int e = 0; e < kUnit; ++e) hits += v[e] >= bound && v[e] != kNegInf;
    }
    if (hits) {
      int at = atomicAdd(&sh.n, hits);
#pragma unroll
      for (int e = 0; e < kUnit; ++e)
        if (v[e] >= bound && v[e] != kNegInf) {
          if (at < kList) sh.l.list[at] = (uint64_t)ord_of(v[e]) << 32 | (uint32_t)~(u * kUnit + e - row.lo);
          ++at;
        }
    }
  }
  __syncthreads();
  return sh.n;
}

// Sorts list[0, n) downwards (the keys differ).
__device__ void sort_down(uint64_t* list, int n) {
  int m = 64;
  while (m < n) m <<= 1;
  for (int i = n + threadIdx.x; i < m; i += kPickThreads) list[i] = 0;
  __syncthreads();
  for (int size = 2; size <= m; size <<= 1)
    for (int d = size >> 1; d > 0; d >>= 1) {
      for (int i = threadIdx.x; i < m / 2; i += kPickThreads) {
        const int x = 2 * i - (i & (d - 1)), y = x + d;
        const uint64_t p = list[x], q = list[y];
        if ((p < q) == ((x & size) == 0)) {
          list[x] = q;
          list[y] = p;
        }
      }
      __syncthreads();
    }
}

__device__ __forceinline__ double z_of(float v, float mx, double inv_t) {
  return ((double)v - (double)mx) * inv_t;
}
// (the largest has weight 1, an infinite one too)
__device__ __forceinline__ double weight(float v, float mx, double inv_t) {
  return v == mx ? 1.0 : weight_of(z_of(v, mx, inv_t));
}
__device__ __forceinline__ double log_prob(float v, float mx, double inv_t, double total) {
  return (v == mx ? 0.0 : z_of(v, mx, inv_t)) - log(total);
}

// Running sums of w[0, n) in place (inclusive), in one order whatever n.
__device__ void running_sums(double* w, int n, PickShared& sh) {
  constexpr int PER = kList / kPickThreads;
  double x[PER], s = 0.0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = threadIdx.x * PER + i;
    x[i] = j < n ? w[j] : 0.0;
    s += x[i];
  }
  double b = block_before(s, sh);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = threadIdx.x * PER + i;
    b += x[i];
    if (j < n) w[j] = b;
  }
  __syncthreads();
}

__device__ __forceinline__ void emit(const SampleArgs& a, int t, int token, double lp) {
  a.token[t] = token;
  if (a.logprob) a.logprob[t] = (float)lp;
}

// The draw among the first n of the sorted list.
__device__ void draw_from_list(const SampleArgs& a, int t, const Params& q, float mx, int n,
                               PickShared& sh) {
  // by index: the key's low half, with the order in place of the high one
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPickThreads) {
    const uint64_t k = sh.l.list[i];
    sh.l.list[i] = k << 32 | k >> 32;
  }
  sort_down(sh.l.list, n);
  for (int i = threadIdx.x; i < n; i += kPickThreads)
    sh.l.w[i] = weight(of_ord((uint32_t)sh.l.list[i]), mx, q.inv_t);
  __syncthreads();
  running_sums(sh.l.w, n, sh);
  const double total = sh.l.w[n - 1], target = q.u * total;
  int before = 0, live = 0;  // sums that do not pass the target; sums below the total
  for (int i = threadIdx.x; i < n; i += kPickThreads) {
    before += sh.l.w[i] <= target;
    live += sh.l.w[i] < total;
  }
  before = block_sum(before, sh);
  live = block_sum(live, sh);
  if (threadIdx.x == 0) {
    const uint64_t k = sh.l.list[before < n ? before : live];
    emit(a, t, (int)~(uint32_t)(k >> 32), log_prob(of_ord((uint32_t)k), mx, q.inv_t, total));
  }
}

// Applies a function to every logit of the row above -inf: f(logit, unit's element).
template <int DT, typename F>
__device__ __forceinline__ void each_logit(const Row& row, F f) {
  const int units = (row.hi + kUnit - 1) / kUnit;
  for (int u = threadIdx.x; u < units; u += kPickThreads) {
    float v[kUnit];
    load_unit<DT>(row, u, v);
#pragma unroll
    for (int e = 0; e < kUnit; ++e)
      if (v[e] != kNegInf) f(v[e], u * kUnit + e);
  }
}

// The bin of the histogram's counts, from the top, in which `need` is reached, and
// the count above it (bin -1: never).
__device__ void count_bin(int need, PickShared& sh, int& bin, int& above) {
  constexpr int PER = kBins / kPickThreads;
  int c[PER], s = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    c[i] = (int)sh.h.count[kBins - 1 - (threadIdx.x * PER + i)];
    s += c[i];
  }
  int b = block_before(s, sh);
  if (threadIdx.x == 0) sh.found = -1;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (b < need && b + c[i] >= need) {
      sh.found = kBins - 1 - (threadIdx.x * PER + i);
      sh.extra = b;
    }
    b += c[i];
  }
  __syncthreads();
  bin = sh.found;
  above = sh.extra;
  __syncthreads();
}

// The k-th largest logit's order, and how many of its equals are among the k (0
// equals: the row has fewer than k logits above -inf).
template <int DT>
__device__ void kth_largest(const Row& row, int k, PickShared& sh, uint32_t& key, int& equals) {
  uint32_t prefix = 0;
  int need = k;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
    const uint32_t bins = pass < 2 ? 0x7ffu : 0x3ffu;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kPickThreads) sh.h.count[i] = 0;
    __syncthreads();
    each_logit<DT>(row, [&](float v, int) {
      const uint32_t o = ord_of(v);
      if (pass == 0 || (o >> (shift + (pass == 1 ? 11 : 10))) == prefix)
        atomicAdd(&sh.h.count[(o >> shift) & bins], 1u);
    });
    __syncthreads();
    int bin, above;
    count_bin(need, sh, bin, above);
    if (bin < 0) {
      key = 0;
      equals = 0;
      return;
    }
    prefix = pass == 0 ? (uint32_t)bin : (prefix << (pass == 1 ? 11 : 10)) | (uint32_t)bin;
    need -= above;
  }
  key = prefix;
  equals = need;
}

// The whole row: cuts it by histograms and draws.  What is kept at the end is
// every logit above `cut`, and the first `equals` of those that equal it.
template <int DT>
__device__ void whole_row(const SampleArgs& a, int t, const Row& row, const Params& q, float mx,
                          PickShared& sh) {
  uint32_t cut = 0;  // (-inf's order and below: nothing equals it)
  int equals = 0;
  if (q.k > 0) {
    kth_largest<DT>(row, q.k, sh, cut, equals);
    // below min_p already: the cut is min_p's
    if (equals && weight(of_ord(cut), mx, q.inv_t) < q.min_p) cut = 0, equals = 0;
  }
  const bool cuts = q.k > 0 || q.p < 1.0 || q.min_p > 0.0;
  auto kept = [&](float v, double w) { return ord_of(v) > cut && w >= q.min_p; };
  if (q.p < 1.0) {
    const double w_cut = equals ? weight(of_ord(cut), mx, q.inv_t) : 0.0;
    double top = 0.0, width = 1.0 / 64.0;  // the bins: [top - (b + 1) width, top - b width)
    double base = 0.0, limit = 0.0;        // weight above the bins; top_p of all
    int count = 0;                         // logits above the bins
    for (int level = 0;; ++level) {
      // (the top is the top of a bin one level up; the last bin of the first level
      // takes everything below, which no top_p reaches)
      const double per = 1.0 / width;
      auto bin_of = [&](float v) {
        const double x = (top - z_of(v, mx, q.inv_t)) * per;
        if (v == mx) return level == 0 || top == 0.0 ? 0 : -1;
        if (level == 0) return x < (double)(kBins - 1) ? (int)x : kBins - 1;
        return x >= 0.0 && x < (double)kBins ? (int)x : -1;
      };
      __syncthreads();
      for (int i = threadIdx.x; i < kBins; i += kPickThreads) {
        sh.h.mass[i] = 0;
        sh.h.count[i] = 0;
      }
      __syncthreads();
      each_logit<DT>(row, [&](float v, int) {
        const int b = bin_of(v);
        if (b < 0) return;
        const double w = v == mx ? 1.0 : weight_of(z_of(v, mx, q.inv_t));
        if (!kept(v, w) || w == 0.0) return;
        // relative to the weight at the bin's top, so that nothing is lost
        const double rel =
            v == mx ? 1.0 : weight_of(fmin(z_of(v, mx, q.inv_t) - (top - b * width), 0.0));
        atomicAdd(&sh.h.count[b], 1u);
        atomicAdd(&sh.h.mass[b], (unsigned long long)(rel * 0x1p42));
      });
      __syncthreads();
      // running sums over the bins; the first with logits that reaches the limit
      constexpr int PER = kBins / kPickThreads;
      double mass[PER], s = 0.0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int b = threadIdx.x * PER + i;
        mass[i] = (double)sh.h.mass[b] * 0x1p-42 * weight_of(top - b * width);
        s += mass[i];
      }
      if (level == 0) limit = q.p * (block_sum(s, sh) + equals * w_cut);
      double m = base + block_before(s, sh);
      if (threadIdx.x == 0) sh.found = kBins;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int b = threadIdx.x * PER + i;
        m += mass[i];
        if (m >= limit && sh.h.count[b] > 0) atomicMin(&sh.found, b);
        sh.h.mass[b] = (unsigned long long)__double_as_longlong(m);
      }
      __syncthreads();
      const int b = sh.found;
      const double all = __longlong_as_double((long long)sh.h.mass[kBins - 1]);
      if (limit <= 0.0) {  // top_p of 0: the first of the largest
        cut = ord_of(mx);
        equals = 1;
        break;
      }
      if (b == kBins) {  // reached among the equals of the cut, or by rounding at the end
        const double c = w_cut > 0.0 ? ceil((limit - all) / w_cut) : 0.0;
        equals = c < (double)equals ? max((int)c, 0) : equals;
        break;
      }
      if (b > 0) base = __longlong_as_double((long long)sh.h.mass[b - 1]);
      const int here = (int)sh.h.count[b];
      {
        int c = 0;
        for (int i = threadIdx.x; i < b; i += kPickThreads) c += (int)sh.h.count[i];
        count += block_sum(c, sh);
      }
      __syncthreads();
      if (here <= kList) {
        if (threadIdx.x == 0) sh.n = 0;
        __syncthreads();
        each_logit<DT>(row, [&](float v, int j) {
          if (bin_of(v) != b) return;
          if (!kept(v, v == mx ? 1.0 : weight_of(z_of(v, mx, q.inv_t)))) return;
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList) sh.l.list[at] = (uint64_t)ord_of(v) << 32 | (uint32_t)~(j - row.lo);
        });
        __syncthreads();
        const int n = min(sh.n, kList);
        sort_down(sh.l.list, n);
        for (int i = threadIdx.x; i < n; i += kPickThreads)
          sh.l.w[i] = weight(of_ord((uint32_t)(sh.l.list[i] >> 32)), mx, q.inv_t);
        __syncthreads();
        running_sums(sh.l.w, n, sh);
        // the last kept one is the first whose running sum reaches the limit
        int before = 0;
        for (int i = threadIdx.x; i < n; i += kPickThreads) before += base + sh.l.w[i] < limit;
        before = min(block_sum(before, sh), n - 1);
        cut = (uint32_t)(sh.l.list[before] >> 32);
        int eq = 0;
        for (int i = threadIdx.x; i <= before; i += kPickThreads)
          eq += (uint32_t)(sh.l.list[i] >> 32) == cut;
        equals = block_sum(eq, sh);
        break;
      }
      // too many to sort: one value, or values whose weights are the same to 2^-50
      if (threadIdx.x == 0) {
        sh.lo = 0xffffffffu;
        sh.hi = 0;
      }
      __syncthreads();
      {
        uint32_t lo = 0xffffffffu, hi = 0;
        each_logit<DT>(row, [&](float v, int) {
          if (bin_of(v) != b) return;
          if (!kept(v, v == mx ? 1.0 : weight_of(z_of(v, mx, q.inv_t)))) return;
          lo = min(lo, ord_of(v));
          hi = max(hi, ord_of(v));
        });
        atomicMin(&sh.lo, lo);
        atomicMax(&sh.hi, hi);
      }
      __syncthreads();
      const uint32_t lo = sh.lo, hi = sh.hi;
      __syncthreads();
      if (lo == hi || level == 4) {
        const double c = ceil((limit - base) / weight(of_ord(hi), mx, q.inv_t));
        const int n = c < 1.0 ? 1 : (c < (double)here ? (int)c : here);
        if (lo == hi) {
          cut = hi;
          equals = n;
        } else {
          kth_largest<DT>(row, count + n, sh, cut, equals);
        }
        break;
      }
      top -= b * width;
      width /= kBins;
    }
  }

  // The draw: blocks' counts of equals of the cut, then their weights.
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per_group = (64 << a.gshift);
  auto block_max = [&](int b) {  // of a block of 512 (at most that many groups)
    float m = kNegInf;
    for (int g = b * kBlock / per_group; g <= (b * kBlock + kBlock - 1) / per_group; ++g)
      if (g < a.ng) m = fmaxf(m, sh.gmax[g]);
    return m;
  };
  __syncthreads();
  for (int b = wave; b < a.nb; b += kPickWaves) {
    int c = 0;
    if (equals && ord_of(block_max(b)) >= cut) {
      float v[kUnit];
      load_unit<DT>(row, b * 64 + lane, v);
#pragma unroll
      for (int e = 0; e < kUnit; ++e) c += v[e] != kNegInf && ord_of(v[e]) == cut;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
    }
    if (lane == 0) sh.b.ties[b] = c;
  }
  __syncthreads();
  {
    constexpr int PER = (kMaxBlocks + kPickThreads - 1) / kPickThreads;
    int c[PER], s = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      c[i] = b < a.nb ? sh.b.ties[b] : 0;
      s += c[i];
    }
    int before = block_before(s, sh);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      if (b < a.nb) sh.b.ties[b] = before;
      before += c[i];
    }
  }
  __syncthreads();
  // a lane's weights of block b
  auto weights = [&](int b, float (&v)[kUnit], double (&w)[kUnit]) {
    load_unit<DT>(row, b * 64 + lane, v);
    int c = 0;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) c += v[e] != kNegInf && ord_of(v[e]) == cut;
    int x = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    int tie = sh.b.ties[b] + x - c;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      const double f = v[e] == kNegInf ? 0.0 : weight(v[e], mx, q.inv_t);
      const bool eq = v[e] != kNegInf && ord_of(v[e]) == cut;
      w[e] = (ord_of(v[e]) > cut || (eq && tie < equals)) && f >= q.min_p ? f : 0.0;
      tie += eq;
    }
  };
  for (int b = wave; b < a.nb; b += kPickWaves) {
    double s = 0.0;
    if (!cuts) {  // every logit is kept: the sums of the first launch
      const float ref = a.bref[(size_t)t * a.nb + b];
      if (lane == 0)
        sh.b.mass[b] =
            ref == kNegInf ? 0.0 : a.bmass[(size_t)t * a.nb + b] * weight(ref, mx, q.inv_t);
      continue;
    }
    const float m = block_max(b);
    if (m != kNegInf && ord_of(m) >= cut) {
      float v[kUnit];
      double w[kUnit];
      weights(b, v, w);
#pragma unroll
      for (int e = 0; e < kUnit; ++e) s += w[e];
      s = wave_sum(s);
    }
    if (lane == 0) sh.b.mass[b] = s;
  }
  __syncthreads();
  double total;
  {
    constexpr int PER = (kMaxBlocks + kPickThreads - 1) / kPickThreads;
    double x[PER], s = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      x[i] = b < a.nb ? sh.b.mass[b] : 0.0;
      s += x[i];
    }
    double before = block_before(s, sh);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      before += x[i];
      if (b < a.nb) sh.b.mass[b] = before;
    }
    __syncthreads();
    total = sh.b.mass[a.nb - 1];
  }
  const double target = q.u * total;
  int first = 0;  // the first block whose running sum passes the target
  for (int b = threadIdx.x; b < a.nb; b += kPickThreads) first += sh.b.mass[b] <= target;
  first = block_sum(first, sh);
  if (wave != 0) return;
  // (the sum within a block may round otherwise: then the next block has it)
  for (int b = first; b < a.nb; ++b) {
    float v[kUnit];
    double w[kUnit], s = 0.0;
    weights(b, v, w);
#pragma unroll
    for (int e = 0; e < kUnit; ++e) s += w[e];
    double x = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    double run = (b ? sh.b.mass[b - 1] : 0.0) + (x - s);
    int hit = -1;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      run += w[e];
      if (hit < 0 && w[e] > 0.0 && run > target) hit = e;
    }
    const uint64_t any = __ballot(hit >= 0);
    if (any) {
      if (lane == (int)__builtin_ctzll(any)) {
#pragma unroll
        for (int e = 0; e < kUnit; ++e)
          if (e == hit)
            emit(a, t, (b * 64 + lane) * kUnit + e - row.lo,
                 log_prob(v[e], mx, q.inv_t, total));
      }
      return;
    }
  }
  // nothing passes (a uniform of 1 or more): the last one with a weight
  for (int b = a.nb - 1; b >= 0; --b) {
    float v[kUnit];
    double w[kUnit];
    weights(b, v, w);
    int hit = -1;
#pragma unroll
    for (int e = 0; e < kUnit; ++e)
      if (w[e] > 0.0) hit = e;
    const uint64_t any = __ballot(hit >= 0);
    if (any) {
      if (lane == 63 - (int)__builtin_clzll(any)) {
#pragma unroll
        for (int e = 0; e < kUnit; ++e)
          if (e == hit)
            emit(a, t, (b * 64 + lane) * kUnit + e - row.lo,
                 log_prob(v[e], mx, q.inv_t, total));
      }
      return;
    }
  }
}

template <int DT>
__global__ __launch_bounds__(kPickThreads) void pick_kernel(SampleArgs a) {
  __shared__ PickShared sh;
  const int t = blockIdx.x;
  const Row row = row_of<DT>(a, t);
  const Params q = params_of(a, t);
  float mx = kNegInf;
  for (int g = threadIdx.x; g < a.ng; g += kPickThreads) {
    const float m = a.gmax[(size_t)t * a.ng + g];
    sh.gmax[g] = m;
    mx = fmaxf(mx, m);
  }
  mx = wave_max(mx);
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = (double)mx;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w) mx = fmaxf(mx, (float)sh.part[w]);
  __syncthreads();
  if (mx == kNegInf) {  // no token
    if (threadIdx.x == 0) emit(a, t, -1, (double)kNegInf);
    return;
  }
  if (q.greedy) {
    const int n = gather<DT>(a, row, mx, sh);  // the largest and its equals
    uint64_t best = 0;
    for (int i = threadIdx.x; i < min(n, kList); i += kPickThreads)
      best = best > sh.l.list[i] ? best : sh.l.list[i];
    if (n > kList) {  // (more equals than the list holds)
      each_logit<DT>(row, [&](float v, int j) {
        const uint64_t k = (uint64_t)ord_of(v) << 32 | (uint32_t)~(j - row.lo);
        best = best > k ? best : k;
      });
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t x = __shfl_xor((unsigned long long)best, o, 64);
      best = best > x ? best : x;
    }
    if ((threadIdx.x & 63) == 0) sh.l.w[threadIdx.x >> 6] = __longlong_as_double((long long)best);
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 0; w < kPickWaves; ++w) {
        const uint64_t x = (uint64_t)__double_as_longlong(sh.l.w[w]);
        best = best > x ? best : x;
      }
      emit(a, t, (int)~(uint32_t)best, 0.0);
    }
    return;
  }
  const bool cuts = q.k > 0 || q.p < 1.0 || q.min_p > 0.0;
  float bound = kNegInf;
  double total = 0.0;  // of all weights, where the row has no other filter than top_p
  bool try_list = a.V <= kList;
  if (bounded(a, q)) {
    if (q.k > 0 && q.k <= a.ng) bound = group_bound(a, q.k, sh);
    if (q.min_p > 0.0) {
      // a little below the logit of weight min_p
      const double v = (double)mx + log(q.min_p) / q.inv_t;
      bound = fmaxf(bound, (float)(v - fabs(v) * 1e-6 - 1e-30));
    }
    try_list = true;
  } else {
    double s = 0.0;
    for (int b = threadIdx.x; b < a.nb; b += kPickThreads) {
      const float ref = a.bref[(size_t)t * a.nb + b];
      s += ref == kNegInf ? 0.0 : a.bmass[(size_t)t * a.nb + b] * weight(ref, mx, q.inv_t);
    }
    total = block_sum(s, sh);
    if (cuts && q.k == 0 && a.V > kList) {
      bound = group_bound(a, min(a.ng, 256), sh);
      try_list = true;
    }
  }
  if (try_list && cuts) {
    const int n = gather<DT>(a, row, bound, sh);
    if (n <= kList) {
      sort_down(sh.l.list, n);
      int fit = 0;  // of at least min_p
      for (int i = threadIdx.x; i < n; i += kPickThreads) {
        const double w = weight(of_ord((uint32_t)(sh.l.list[i] >> 32)), mx, q.inv_t);
        sh.l.w[i] = w;
        fit += w >= q.min_p;
      }
      int m = max(block_sum(fit, sh), 1);
      if (q.k > 0) m = min(m, q.k);
      bool done = true;
      if (q.p < 1.0) {
        running_sums(sh.l.w, m, sh);
        const double sum = sh.l.w[m - 1];
        // only top_p, and logits outside the list: its sum is that of the row
        const bool open = !bounded(a, q) && a.V > kList;
        const double limit = q.p * (open ? total : sum);
        done = !open || sum >= limit;
        int kept = 0;
        for (int i = threadIdx.x; i < m; i += kPickThreads)
          kept += (i ? sh.l.w[i - 1] : 0.0) < limit;
        m = max(block_sum(kept, sh), 1);
      }
      if (done) {
        draw_from_list(a, t, q, mx, m, sh);
        return;
      }
    }
  }
  whole_row<DT>(a, t, row, q, mx, sh);
}

template <int DT>
hipError_t launch(const SampleArgs& a, hipStream_t stream) {
  constexpr int W = kScanThreads / 64;
  // few rows: more workgroups of less each
  const int bpw = (long long)a.T * a.nb < 4096 * W ? 2 : 8;
  const int segs = (a.nb + W * bpw - 1) / (W * bpw);
  if (bpw == 2)
    scan_kernel<DT, 2><<<(unsigned)(a.T * segs), kScanThreads, 0, stream>>>(a, segs);
  else
    scan_kernel<DT, 8><<<(unsigned)(a.T * segs), kScanThreads, 0, stream>>>(a, segs);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pick_kernel<DT><<<(unsigned)a.T, kPickThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

void plan_sample(int V, int* ng, int* nb, int* gshift) {
  const int span = V + kUnit - 1;  // elements from the 16-byte boundary on
  int s = 0;
  while ((span + (64 << s) - 1) / (64 << s) > kMaxGroups - 1) ++s;
  *gshift = s;
  *ng = (span + (64 << s) - 1) / (64 << s);
  *nb = (span + kBlock - 1) / kBlock;
}

size_t sample_bytes(int T, int V) {
  int ng, nb, s;
  plan_sample(V, &ng, &nb, &s);
  return ((size_t)T * ((size_t)nb * 12 + (size_t)ng * 4) + 511) / 256 * 256;
}

void place_sample(SampleArgs* a, void* workspace) {
  plan_sample(a->V, &a->ng, &a->nb, &a->gshift);
  a->bmass = (double*)workspace;
  a->bref = (float*)(a->bmass + (size_t)a->T * a->nb);
  a->gmax = a->bref + (size_t)a->T * a->nb;
}

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PCTREE_F32: return launch<PCTREE_F32>(a, stream);
    case PCTREE_BF16: return launch<PCTREE_BF16>(a, stream);
    default: return launch<PCTREE_F16>(a, stream);
  }
}

}  // namespace pctree
