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
// scan_kernel reads the logits once: maxima of groups of 8 to 512 logits (at most
// 2560 of a row), and for the rows that need all of it (no top_k, no min_p) the sum
// of weights of each block of 512.  pick_kernel, one workgroup a row, starts from
// those.  The k-th largest of maxima over disjoint parts of the row is a lower bound
// of the k-th largest logit, so only groups that reach it are read again, and what
// reaches it, hardly more than k logits, is sorted in LDS; min_p gives such a bound
// too, and a top_p alone first tries the logits from the 256-th largest maximum up.
// A row without filters needs only the blocks' sums and the one block that the draw
// falls into.
//
// Open rows, where top_p or min_p keeps more than that, are left to three more launches
// over all compute units: hist_kernel sums the weights in bins of 1/64 in log
// weight, mark_kernel finds the bin in which top_p is reached, sums each block's
// weights above it and lists the bin's own logits, and finish_kernel cuts that list
// and draws.  One workgroup could do it alone (whole_row; it does for a top_k that the
// bounds or the list do not reach, and where the bin's list does not do), which takes
// several times as long.
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

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
constexpr int kParts = 512;           // parts of a row whose maxima bound its k-th largest logit,
constexpr int kManyParts = 2048;      // ... and where k is more than a quarter of that
constexpr int kMaxBound = 1024;       // the largest k that is bounded so
// (top_p alone) the rank of the bound that is tried first.  One row of 150,000 logits that
// keeps 70 of them: 32 us, 30 with 128, 43 with 512; one that keeps 640, open with each:
// 53, 50, 42; rows that keep 130 to 250 need 256.
constexpr int kTry = 256;
constexpr int kBins = 2048;           // of 1/64 in log weight
// A row that filters by weight alone with more groups than this in reach of its bound is
// left to the open rows' launches at once (up to 768 groups: 512 rows' picks 42 us, 33; they
// would read as much as those do, one workgroup a row).
constexpr int kFewGroups = 400;
constexpr int kOpenGrid = 1024;       // workgroups that share the open rows' items
constexpr double kBinStep = 0.98449643700540841;  // e^(-1/64)
constexpr double kLowest = -700.0;    // weights below e^-700 are 0
constexpr double kLog2e = 1.4426950408889634074;

// 2^r, |r| <= 1/2, by its Taylor series (the first term left out, the thirteenth, is below 2^-52).
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
// e^z for z in [-700, 0]; 0 below (and for NaN).  The whole part of the exponent is the
// low bits of a float64 of step 1, and is added to the result's exponent (2^-1010 is
// still normal): no conversions, which take four times a product's time.
__device__ __forceinline__ double weight_of(double z) {
  constexpr double kStep = 0x1.8p52;
  const double t = z * kLog2e, n = t + kStep;
  const double p = exp2_small(t - (n - kStep));
  const uint32_t lo = (uint32_t)__double_as_longlong(n);
  const uint64_t bits = (uint64_t)__double_as_longlong(p);
  const double w = __longlong_as_double(
      (long long)((uint64_t)((uint32_t)(bits >> 32) + (lo << 20)) << 32 | (uint32_t)bits));
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

// A logit and its index as one number: larger logits first, then lower indices.
__device__ __forceinline__ uint64_t key_of(float v, int i) {
  return (uint64_t)ord_of(v) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float logit_of(uint64_t key) { return of_ord((uint32_t)(key >> 32)); }
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }

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
// (a unit's bytes, as loaded)
template <int DT>
struct Raw {
  u32x4 x[DT == PCTREE_F32 ? 2 : 1];
};
// (A unit that is not all inside the row is put together from its elements, -inf
// elsewhere; in a loop, since code that runs once costs its fetch: 0.1 us a line.)
template <int DT>
__device__ __forceinline__ Raw<DT> load_raw(const Row& r, int u) {
  Raw<DT> w;
  constexpr int N = DT == PCTREE_F32 ? 2 : 1;
  const int j0 = u * kUnit;
  if (j0 >= r.lo && j0 + kUnit <= r.hi) {
#pragma unroll
    for (int i = 0; i < N; ++i) w.x[i] = ((const u32x4*)r.base)[(size_t)u * N + i];
    return w;
  }
  constexpr uint32_t low = DT == PCTREE_F32 ? 0xff800000u : (DT == PCTREE_F16 ? 0xfc00fc00u : 0xff80ff80u);
#pragma unroll
  for (int i = 0; i < N; ++i) w.x[i] = u32x4{low, low, low, low};
#pragma unroll 1
  for (int j = max(j0, r.lo); j < min(j0 + kUnit, r.hi); ++j) {
    const int e = j - j0;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      const uint32_t x = w.x[i / 4][i % 4];
      if constexpr (DT == PCTREE_F32) {
        w.x[i / 4][i % 4] = i == e ? ((const uint32_t*)r.base)[j] : x;
      } else {
        const uint32_t h = ((const uint16_t*)r.base)[j];
        w.x[i / 4][i % 4] =
            i == e / 2 ? (e & 1 ? (x & 0xffffu) | h << 16 : (x & 0xffff0000u) | h) : x;
      }
    }
  }
  return w;
}
// A queue of raws: drops the first, appends one.  (A loop that takes the first each
// time has one copy of its body; indexing registers would need one each.)
template <int DT, int N>
__device__ __forceinline__ void next_raw(Raw<DT> (&w)[N], const Raw<DT>& x) {
#pragma unroll
  for (int i = 0; i + 1 < N; ++i) w[i] = w[i + 1];
  w[N - 1] = x;
}
template <int DT, bool MEND = true>
__device__ __forceinline__ void unpack(const Raw<DT>& w, float (&v)[kUnit]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (DT == PCTREE_F32) {
      v[e] = __uint_as_float(w.x[0][e]);
      v[4 + e] = __uint_as_float(w.x[1][e]);
    } else {
      v[2 * e] = lo16<DT == PCTREE_F16>(w.x[0][e]);
      v[2 * e + 1] = hi16<DT == PCTREE_F16>(w.x[0][e]);
    }
  }
  if constexpr (MEND) {
#pragma unroll
    for (int e = 0; e < kUnit; ++e) v[e] = v[e] == v[e] ? v[e] : kNegInf;
  }
}
template <int DT>
__device__ __forceinline__ void load_unit(const Row& r, int u, float (&v)[kUnit]) {
  unpack<DT>(load_raw<DT>(r, u), v);
}
// The units u0 + 64 i + lane, i < N, of a wave: all loads before the first use where
// the wave is inside the row.
template <int DT, int N>
__device__ __forceinline__ void load_raws(const Row& r, int u0, Raw<DT> (&w)[N]) {
  const int lane = threadIdx.x & 63;
  if (u0 * kUnit >= r.lo && (u0 + 64 * N) * kUnit <= r.hi) {
    constexpr int X = DT == PCTREE_F32 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < X; ++j)
        w[i].x[j] = ((const u32x4*)r.base)[(size_t)(u0 + 64 * i + lane) * X + j];
    return;
  }
#pragma unroll 1
  for (int i = 0; i < N; ++i) {
    const Raw<DT> x = load_raw<DT>(r, u0 + 64 * i + lane);
    next_raw(w, x);
  }
}

// A row's parameters.
struct Params {
  double inv_t, p, min_p, u;
  int k;        // 0: off
  bool greedy;  // a temperature of 0 (or below, or NaN): the largest logit
};
// (Absent arrays point at `uniform`, so that all loads are issued together.)
__device__ __forceinline__ Params params_of(const SampleArgs& a, int t) {
  const float T = a.temperature[t], p = a.top_p[t], m = a.min_p[t], u = a.uniform[t];
  const int k = a.top_k[t];
  Params q;
  q.greedy = (a.has & kHasTemperature) && !(T > 0.0f);
  q.inv_t = q.greedy || !(a.has & kHasTemperature) ? 1.0 : 1.0 / (double)T;
  q.k = (a.has & kHasTopK) && k > 0 && k < a.V ? k : 0;
  q.p = (a.has & kHasTopP) && p < 1.0f ? (double)p : 1.0;  // (NaN: off)
  q.min_p = (a.has & kHasMinP) && m > 0.0f ? (double)fminf(m, 1.0f) : 0.0;
  // (1 and more: infinite, so that no running sum passes it, however that was rounded)
  q.u = u >= 1.0f ? (double)__builtin_inff() : (u > 0.0f ? (double)u : 0.0);
  return q;
}
// Whether the row is settled from its largest logits, without the sum of all.
__device__ __forceinline__ bool bounded(const SampleArgs& a, const Params& q) {
  return q.greedy || q.min_p > 0.0 || (q.k > 0 && q.k <= min(a.ng, kMaxBound));
}

// The value of the lane whose index differs in bit D (row operations and lane swaps:
// a tenth of the latency of an exchange through LDS).
template <int D>
__device__ __forceinline__ uint32_t xor_lane(uint32_t x) {
  if constexpr (D == 1) return __builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true);
  if constexpr (D == 2) return __builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true);
  if constexpr (D == 4)  // (7 - i in each eight, then 3 - i in each four)
    return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true), 0x1b,
                                    0xf, 0xf, true);
  if constexpr (D == 8) return __builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true);
  if constexpr (D == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? s[0] : s[1];
  }
  const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return threadIdx.x & 32 ? s[0] : s[1];
}
template <int D>
__device__ __forceinline__ uint64_t xor_lane(uint64_t x) {
  return (uint64_t)xor_lane<D>((uint32_t)(x >> 32)) << 32 | xor_lane<D>((uint32_t)x);
}
template <int D>
__device__ __forceinline__ double xor_lane(double x) {
  return __longlong_as_double((long long)xor_lane<D>((uint64_t)__double_as_longlong(x)));
}

// Sums over the lanes up to each one (its own among them), and over the wave: row
// shifts by 1, 2, 4, 8, then the rows' last lanes into the rows after them.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_from(int x) {  // (0 where there is no such lane)
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_from(double x) {
  const long long b = __double_as_longlong(x);
  const uint32_t hi = (uint32_t)dpp_from<CTRL, ROWS>((int)(b >> 32)), lo = (uint32_t)dpp_from<CTRL, ROWS>((int)b);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
template <typename T>
__device__ __forceinline__ T wave_upto(T x) {
  x += dpp_from<0x111, 0xf>(x);
  x += dpp_from<0x112, 0xf>(x);
  x += dpp_from<0x114, 0xf>(x);
  x += dpp_from<0x118, 0xf>(x);
  x += dpp_from<0x142, 0xa>(x);
  x += dpp_from<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ uint32_t wave_most(uint32_t x) {
  auto step = [&](uint32_t y) { x = max(x, y); };
  step(xor_lane<1>(x));
  step(xor_lane<2>(x));
  step(xor_lane<4>(x));
  step(xor_lane<8>(x));
  step(xor_lane<16>(x));
  step(xor_lane<32>(x));
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ int wave_count(int x) {
  return __builtin_amdgcn_readlane(wave_upto(x), 63);
}
__device__ __forceinline__ uint64_t lane_of(uint64_t x, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  return __longlong_as_double((long long)lane_of((uint64_t)__double_as_longlong(x), lane));
}
__device__ __forceinline__ double wave_sum(double v) {
  v += xor_lane<32>(v);
  v += xor_lane<16>(v);
  v += xor_lane<8>(v);
  v += xor_lane<4>(v);
  v += xor_lane<2>(v);
  v += xor_lane<1>(v);
  return v;
}

// The sums of N values over the wave, N a power of two: lane l gets that of value l /
// (64 / N).  Halves of the values go to the lanes' halves first.
template <int N, int D = 32>
__device__ __forceinline__ double wave_sums(double (&v)[N]) {
  if constexpr (N == 1) {
    double x = v[0];
    if constexpr (D >= 32) x += xor_lane<32>(x);
    if constexpr (D >= 16) x += xor_lane<16>(x);
    if constexpr (D >= 8) x += xor_lane<8>(x);
    if constexpr (D >= 4) x += xor_lane<4>(x);
    if constexpr (D >= 2) x += xor_lane<2>(x);
    if constexpr (D >= 1) x += xor_lane<1>(x);
    return x;
  } else {
    double h[N / 2];
    const bool upper = threadIdx.x & D;
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
      h[i] = (upper ? v[i + N / 2] : v[i]) + xor_lane<D>(upper ? v[i] : v[i + N / 2]);
    return wave_sums<N / 2, D / 2>(h);
  }
}

// Bytes bound it where rows filter: 512 bf16 rows of 151936, 156 MB, in 43 us (3.6 TB/s); 3
// us for one row.  Where no row does, the float64 exponentials of all weights do: 98 us.
template <int DT, int BPW>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(SampleArgs a, int segs) {
  const int t = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int lane = threadIdx.x & 63;
  const int b0 = (seg * (kScanThreads / 64) + threadIdx.x / 64) * BPW;
  if (a.open_n && blockIdx.x == 0 && threadIdx.x == 0) *a.open_n = 0;
  if (b0 >= a.nb) return;
  const Row row = row_of<DT>(a, t);
  Raw<DT> raw[BPW];
  load_raws<DT, BPW>(row, b0 * 64, raw);
  const Params q = params_of(a, t);
  const int s = a.gshift;  // a group is the units of 1 << s lanes
  float all = kNegInf;
#pragma unroll
  for (int i = 0; i < BPW; ++i) {
    float v[kUnit];
    unpack<DT, false>(raw[i], v);  // (a maximum passes over NaN by itself)
    float m = v[0];
#pragma unroll
    for (int e = 1; e < kUnit; ++e) m = fmaxf(m, v[e]);
    m = m == m ? m : kNegInf;
    auto join = [&](uint32_t o) { m = fmaxf(m, __uint_as_float(o)); };
    if (s >= 1) join(xor_lane<1>(__float_as_uint(m)));
    if (s >= 2) join(xor_lane<2>(__float_as_uint(m)));
    if (s >= 3) join(xor_lane<4>(__float_as_uint(m)));
    if (s >= 4) join(xor_lane<8>(__float_as_uint(m)));
    if (s >= 5) join(xor_lane<16>(__float_as_uint(m)));
    if (s >= 6) join(xor_lane<32>(__float_as_uint(m)));
    all = fmaxf(all, m);
    const int g = ((b0 + i) * 64 + lane) >> s;
    if ((lane & ((1 << s) - 1)) == 0 && g < a.ng) a.gmax[(size_t)t * a.ng + g] = m;
  }
  if (bounded(a, q)) return;
  const float ref = of_ord(wave_most(ord_of(all)));
  double sums[BPW];
#pragma unroll 1
  for (int i = 0; i < BPW; ++i) {
    float v[kUnit];
    unpack<DT, false>(raw[0], v);
    next_raw(raw, raw[0]);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      const double w = weight_of(((double)v[e] - (double)ref) * q.inv_t);  // (NaN: 0)
      sum += v[e] == ref ? 1.0 : w;
    }
#pragma unroll
    for (int j = 0; j + 1 < BPW; ++j) sums[j] = sums[j + 1];
    sums[BPW - 1] = sum;
  }
  const double sum = wave_sums<BPW>(sums);
  const int b = b0 + lane / (64 / BPW);
  if (lane % (64 / BPW) == 0 && b < a.nb) {
    a.bmass[(size_t)t * a.nb + b] = ref == kNegInf ? 0.0 : sum;
    a.bref[(size_t)t * a.nb + b] = ref;
  }
}

// ---------------------------------------------------------------------------
// pick: one workgroup a row
// ---------------------------------------------------------------------------

struct PickShared {
  float gmax[6 * kPickThreads];  // (of which kMaxGroups are used)
  union {
    struct {
      union {
        uint64_t list[kList];
        int ties[kMaxBlocks + 1];  // per block
      };
      double w[kMaxBlocks + 1];  // of the list; blocks' sums
    } l;
    struct {
      unsigned long long mass[kBins];
      uint32_t count[kBins];
    } h;
  };
  uint16_t group[kMaxGroups + 3];
  double part[kPickWaves];
  int parti[kPickWaves];
  int counts[3][kPickWaves];
  int n, groups, found, extra;
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
  v = wave_count(v);
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
  const double x = wave_upto(v);
  __syncthreads();
  if (lane == 63) sh.part[wave] = x;
  __syncthreads();
  // (the lane before: wave_shr:1)
  double base = dpp_from<0x138, 0xf>(x);
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w) base += w < wave ? sh.part[w] : 0.0;
  return base;
}
__device__ __forceinline__ int block_before(int v, PickShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int x = wave_upto(v);
  __syncthreads();
  if (lane == 63) sh.parti[wave] = x;
  __syncthreads();
  int base = x - v;
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w) base += w < wave ? sh.parti[w] : 0;
  return base;
}

// A lower bound of the row's j-th largest logit, j <= min(groups, kMaxBound): the j-th
// largest of the maxima of parts of the row, its order's low 12 bits rounded down.
// With P parts and logits in any order about P log(P / (P - j)) logits reach it: 52 of
// 512 parts for j = 50, 450 of 2048 for j = 400 (777 with 512).  The search is by bits,
// from the first in which the largest and the smallest maximum differ: 512 parts by
// each wave for itself, 8 to a lane; 2048 by the workgroup, 4 to a thread.
template <int P>
__device__ __forceinline__ float rank_bound(const SampleArgs& a, int j, float mx, PickShared& sh) {
  constexpr bool ALONE = P == kParts;
  constexpr int N = ALONE ? P / 64 : P / kPickThreads, STEP = ALONE ? 64 : kPickThreads;
  const int at = ALONE ? threadIdx.x & 63 : threadIdx.x;
  uint32_t o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float m = kNegInf;
    for (int g = i * STEP + at; g < a.ng; g += P) m = fmaxf(m, sh.gmax[g]);
    o[i] = ord_of(m);
  }
  uint32_t least = o[0];
#pragma unroll
  for (int i = 1; i < N; ++i) least = min(least, o[i]);
  least = ~wave_most(~least);
  if constexpr (!ALONE) {
    if ((threadIdx.x & 63) == 0) sh.counts[0][threadIdx.x >> 6] = (int)least;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) least = min(least, (uint32_t)sh.counts[0][w]);
  }
  const uint32_t most = ord_of(mx);
  const int top = least == most ? 11 : 31 - __builtin_clz(least ^ most);
  uint32_t lo = most & ~((2u << top) - 1);  // at least j maxima are >= lo
  for (int bit = top; bit >= 12; --bit) {
    const uint32_t mid = lo | (1u << bit);
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c += o[i] >= mid;
    c = wave_count(c);
    if constexpr (!ALONE) {  // (two places in turn: one barrier a step)
      int* counts = sh.counts[1 + (bit & 1)];
      if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = c;
      __syncthreads();
      c = 0;
#pragma unroll
      for (int w = 0; w < kPickWaves; ++w) c += counts[w];
    }
    if (c >= j) lo = mid;
    if (c >= j && c <= j + j / 8 + 2) break;  // (close enough)
  }
  return lo < 0x00800000u ? kNegInf : of_ord(lo);
}
__device__ __forceinline__ float bound_of(const SampleArgs& a, int j, float mx, PickShared& sh) {
  return j <= kParts / 4 ? rank_bound<kParts>(a, j, mx, sh) : rank_bound<kManyParts>(a, j, mx, sh);
}

// Logits >= bound into the list (unordered), as (order, lowest index first);
// returns how many there are (more than kList: not all are in the list).
// (More than `most` groups are not looked at: kList + 1.)
template <int DT>
__device__ int gather(const SampleArgs& a, const Row& row, float bound, int most, PickShared& sh) {
  constexpr int B = 4;  // units whose loads are in flight together
  if (threadIdx.x == 0) sh.n = sh.groups = 0;
  __syncthreads();
  {
    constexpr int N = (kMaxGroups + kPickThreads - 1) / kPickThreads;
    uint32_t in = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = i * kPickThreads + threadIdx.x;
      in |= g < a.ng && sh.gmax[g] >= bound ? 1u << i : 0u;
    }
    const int c = __builtin_popcount(in), upto = wave_upto(c);
    int at = 0;
    if ((threadIdx.x & 63) == 63 && upto) at = atomicAdd(&sh.groups, upto);
    at = __builtin_amdgcn_readlane(at, 63) + upto - c;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (in >> i & 1) sh.group[at++] = (uint16_t)(i * kPickThreads + threadIdx.x);
  }
  __syncthreads();
  if (sh.groups > most) return kList + 1;
  const int per = 1 << a.gshift, units = sh.groups << a.gshift;
  for (int i1 = 0; i1 < units; i1 += B * kPickThreads) {
    const int i0 = i1 + threadIdx.x;
    Raw<DT> raw[B];
    auto unit = [&](int k) {  // (past the end: a unit outside the row)
      const int i = i0 + k * kPickThreads;
      return i < units ? sh.group[i >> a.gshift] * per + (i & (per - 1)) : row.hi / kUnit + 1;
    };
#pragma unroll
    for (int k = 0; k < B; ++k) raw[k] = load_raw<DT>(row, unit(k));
#pragma unroll 1
    for (int k = 0; k < B; ++k) {
      float v[kUnit];
      unpack<DT>(raw[0], v);
      next_raw(raw, raw[0]);
      uint32_t hits = 0;
#pragma unroll
      for (int e = 0; e < kUnit; ++e)
        hits |= v[e] >= bound && v[e] != kNegInf ? 1u << e : 0u;
      if (!__any(hits)) continue;
      // the lane's place: one atomic for the wave
      const int c = __builtin_popcount(hits), upto = wave_upto(c), u = unit(k);
      int at = 0;
      if ((threadIdx.x & 63) == 63) at = atomicAdd(&sh.n, upto);
      at = __builtin_amdgcn_readlane(at, 63) + upto - c;
#pragma unroll
      for (int e = 0; e < kUnit; ++e)
        if (hits >> e & 1) {
          if (at < kList) sh.l.list[at] = key_of(v[e], u * kUnit + e - row.lo);
          ++at;
        }
    }
  }
  __syncthreads();
  return sh.n;
}

// Sorts list[0, n) downwards (the keys differ), n <= E * kPickThreads: a bitonic
// network whose element e * kPickThreads + tid is register e of thread tid.  Distances
// below 64 go between lanes, up to kPickThreads through LDS, above between registers.
template <int E>
__device__ void sort_network(uint64_t* list, int n) {
  uint64_t r[E];
  const int tid = threadIdx.x;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e * kPickThreads + tid;
    r[e] = i < n ? list[i] : 0;
  }
  int m = 64;
  while (m < n) m <<= 1;
  auto keep = [&](int e, uint64_t other, int d, int size) {
    const int i = e * kPickThreads + tid;
    const bool larger = ((i & d) == 0) == ((i & size) == 0);
    r[e] = (other > r[e]) == larger ? other : r[e];
  };
#pragma unroll 1
  for (int size = 2; size <= m; size <<= 1) {
    if constexpr (E >= 2) {
#pragma unroll
      for (int dr = E / 2; dr > 0; dr >>= 1) {
        const int d = dr * kPickThreads;
        if (d < size) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if ((e & dr) == 0) {
              const uint64_t x = r[e], y = r[e + dr];
              keep(e, y, d, size);
              keep(e + dr, x, d, size);
            }
        }
      }
    }
#pragma unroll 1
    for (int d = min(size, kPickThreads) >> 1; d >= 64; d >>= 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) list[e * kPickThreads + tid] = r[e];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) keep(e, list[e * kPickThreads + (tid ^ d)], d, size);
    }
    auto lanes = [&](auto dist) {
      constexpr int d = decltype(dist)::value;
      if (d < size) {
#pragma unroll
        for (int e = 0; e < E; ++e) keep(e, xor_lane<d>(r[e]), d, size);
      }
    };
    lanes(std::integral_constant<int, 32>());
    lanes(std::integral_constant<int, 16>());
    lanes(std::integral_constant<int, 8>());
    lanes(std::integral_constant<int, 4>());
    lanes(std::integral_constant<int, 2>());
    lanes(std::integral_constant<int, 1>());
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e * kPickThreads + tid;
    if (i < n) list[i] = r[e];
  }
  __syncthreads();
}
__device__ __forceinline__ void sort_down(uint64_t* list, int n) {
  static_assert(kList == 4 * kPickThreads, "the largest network");
  __syncthreads();
  if (n <= kPickThreads)
    sort_network<1>(list, n);
  else
    sort_network<4>(list, n);
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

// Sorts the first n of the list and returns the key of the last kept one: the first
// whose running sum of weights, from `base` on, reaches the limit.
__device__ uint64_t last_of_list(int n, double base, double limit, float mx, const Params& q,
                                 PickShared& sh) {
  sort_down(sh.l.list, n);
  for (int i = threadIdx.x; i < n; i += kPickThreads)
    sh.l.w[i] = weight(logit_of(sh.l.list[i]), mx, q.inv_t);
  __syncthreads();
  running_sums(sh.l.w, n, sh);
  int before = 0;
  for (int i = threadIdx.x; i < n; i += kPickThreads) before += base + sh.l.w[i] < limit;
  before = min(block_sum(before, sh), n - 1);
  return sh.l.list[before];
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
  int at = 0;  // sums that do not pass the target
  for (int i = threadIdx.x; i < n; i += kPickThreads) at += sh.l.w[i] <= target;
  at = block_sum(at, sh);
  if (at == n) {  // (a uniform of 1) the last of positive weight, which the sums may have lost
    uint32_t last = 0;
    for (int i = threadIdx.x; i < n; i += kPickThreads)
      if (weight(of_ord((uint32_t)sh.l.list[i]), mx, q.inv_t) > 0.0) last = (uint32_t)i;
    last = wave_most(last);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.parti[threadIdx.x >> 6] = (int)last;
    __syncthreads();
    at = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) at = max(at, sh.parti[w]);
  }
  if (threadIdx.x == 0) {
    const uint64_t k = sh.l.list[at];
    emit(a, t, (int)~(uint32_t)(k >> 32), log_prob(of_ord((uint32_t)k), mx, q.inv_t, total));
  }
}

// The draw by blocks: sh.l.w[b] holds the kept weights of block b.  keep(logit,
// index, weight) says what is kept.
template <int DT, typename F>
__device__ void draw_from_blocks(const SampleArgs& a, int t, const Row& row, const Params& q,
                                 float mx, PickShared& sh, F keep) {
  constexpr int PER = (kMaxBlocks + kPickThreads - 1) / kPickThreads;
  const int lane = threadIdx.x & 63;
  __syncthreads();
  {
    double x[PER], s = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      x[i] = b < a.nb ? sh.l.w[b] : 0.0;
      s += x[i];
    }
    double before = block_before(s, sh);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      before += x[i];
      if (b < a.nb) sh.l.w[b] = before;
    }
  }
  __syncthreads();
  const double total = sh.l.w[a.nb - 1], target = q.u * total;
  int first = 0;  // the first block whose running sum passes the target
  for (int b = threadIdx.x; b < a.nb; b += kPickThreads) first += sh.l.w[b] <= target;
  first = block_sum(first, sh);
  if (threadIdx.x >= 64) return;
  // Block by block from there (the sum within a block may round otherwise, then the
  // next one has it); where nothing passes (a uniform of 1), the last one of positive
  // weight.
  for (int step = 0; step < 2 * a.nb; ++step) {
    const bool back = first + step >= a.nb;
    const int b = back ? 2 * a.nb - 1 - (first + step) : first + step;
    if (b < 0) break;
    float v[kUnit];
    double w[kUnit], s = 0.0;
    load_unit<DT>(row, b * 64 + lane, v);
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      const double f = v[e] == kNegInf ? 0.0 : weight(v[e], mx, q.inv_t);
      w[e] = v[e] != kNegInf && keep(v[e], (b * 64 + lane) * kUnit + e - row.lo, f) ? f : 0.0;
      s += w[e];
    }
    double x = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    double run = (b ? sh.l.w[b - 1] : 0.0) + (x - s);
    int hit = -1;
    float hv = 0.0f;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      run += w[e];
      if (w[e] > 0.0 && (back || (hit < 0 && run > target))) {
        hit = e;
        hv = v[e];
      }
    }
    const uint64_t any = __ballot(hit >= 0);
    if (!any) continue;
    if (lane == (back ? 63 - (int)__builtin_clzll(any) : (int)__builtin_ctzll(any)))
      emit(a, t, (b * 64 + lane) * kUnit + hit - row.lo, log_prob(hv, mx, q.inv_t, total));
    return;
  }
}

// Applies f(logit, index) to every logit of the row above -inf.
template <int DT, typename F>
__device__ __forceinline__ void each_logit(const Row& row, F f) {
  const int units = (row.hi + kUnit - 1) / kUnit;
  for (int u = threadIdx.x; u < units; u += kPickThreads) {
    float v[kUnit];
    load_unit<DT>(row, u, v);
#pragma unroll
    for (int e = 0; e < kUnit; ++e)
      if (v[e] != kNegInf) f(v[e], u * kUnit + e - row.lo);
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
#pragma unroll 1
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

// The key of the n-th logit, by index, of those whose order is `cut` (n >= 1, and
// there are that many).
template <int DT>
__device__ uint64_t nth_equal(const SampleArgs& a, const Row& row, uint32_t cut, int n,
                              PickShared& sh) {
  const int lane = threadIdx.x & 63;
  auto equal_in = [&](int b, int (&eq)[kUnit]) {
    float v[kUnit];
    load_unit<DT>(row, b * 64 + lane, v);
    int c = 0;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      eq[e] = v[e] != kNegInf && ord_of(v[e]) == cut;
      c += eq[e];
    }
    return c;
  };
  __syncthreads();
  for (int b = threadIdx.x >> 6; b < a.nb; b += kPickWaves) {
    int eq[kUnit];
    int c = equal_in(b, eq);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
    if (lane == 0) sh.l.ties[b] = c;
  }
  __syncthreads();
  constexpr int PER = (kMaxBlocks + kPickThreads - 1) / kPickThreads;
  int c[PER], s = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    c[i] = b < a.nb ? sh.l.ties[b] : 0;
    s += c[i];
  }
  int before = block_before(s, sh);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < n && before + c[i] >= n) {
      sh.found = threadIdx.x * PER + i;
      sh.extra = before;
    }
    before += c[i];
  }
  __syncthreads();
  const int b = sh.found;
  int need = n - sh.extra;
  int eq[kUnit];
  int x = equal_in(b, eq);
  need += x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  need -= x;  // (of the lane's own)
  if (threadIdx.x < 64) {
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      need -= eq[e];
      if (eq[e] && need == 0) sh.extra = (b * 64 + lane) * kUnit + e - row.lo;
    }
  }
  __syncthreads();
  const int at = sh.extra;
  __syncthreads();
  return (uint64_t)cut << 32 | (uint32_t)~at;
}

// The whole row by one workgroup: cuts it by histograms and draws.  What is kept at
// the end is every logit whose key is at least `last`.  (A top_k of 2000 over 150,000
// logits takes it: 241 us a call of one row, 508 of 512.)
template <int DT>
__device__ __noinline__ void whole_row(const SampleArgs& a, int t, const Row& row, const Params& q,
                                       float mx, PickShared& sh) {
  uint64_t last = 0;
  uint32_t cut = 0;  // logits above it, and the first `equals` of those that equal it
  int equals = 0;
  if (q.k > 0) {
    kth_largest<DT>(row, q.k, sh, cut, equals);
    // below min_p already: the cut is min_p's
    if (equals && weight(of_ord(cut), mx, q.inv_t) < q.min_p) cut = 0, equals = 0;
  }
  auto kept = [&](float v, double w) { return ord_of(v) > cut && w >= q.min_p; };
  if (q.p < 1.0) {
    const double w_cut = equals ? weight(of_ord(cut), mx, q.inv_t) : 0.0;
    double top = 0.0, width = 1.0 / 64.0;  // the bins: [top - (b + 1) width, top - b width)
    double base = 0.0, limit = 0.0;        // weight above the bins; top_p of all
    int count = 0;                         // logits above the bins
#pragma unroll 1
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
        const double w = weight(v, mx, q.inv_t);
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
      uint32_t first = 0;  // the complement of the thread's first such bin
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int b = threadIdx.x * PER + i;
        m += mass[i];
        if (m >= limit && sh.h.count[b] > 0) first = max(first, ~(uint32_t)b);
        sh.h.mass[b] = (unsigned long long)__double_as_longlong(m);
      }
      first = wave_most(first);
      if ((threadIdx.x & 63) == 0 && first) atomicMin(&sh.found, (int)~first);
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
        // (fewer than one: the logits above the cut reach it)
        if (equals && c < (double)equals) equals = max((int)c, 0);
        if (equals == 0 && cut) cut += 1;
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
        each_logit<DT>(row, [&](float v, int i) {
          const bool in = bin_of(v) == b && kept(v, weight(v, mx, q.inv_t));
          const uint64_t all_in = __ballot(in);
          if (!in) return;
          // (the first of them takes the places)
          const int lane = threadIdx.x & 63, lead = (int)__builtin_ctzll(all_in);
          int at = 0;
          if (lane == lead) at = atomicAdd(&sh.n, __builtin_popcountll(all_in));
          at = __builtin_amdgcn_readlane(at, lead) + __builtin_popcountll(all_in & ((1ull << lane) - 1));
          if (at < kList) sh.l.list[at] = key_of(v, i);
        });
        __syncthreads();
        last = last_of_list(min(sh.n, kList), base, limit, mx, q, sh);
        equals = -1;  // (known)
        break;
      }
      // too many to sort: one value, or values whose weights are the same to 2^-45
      if (threadIdx.x == 0) {
        sh.lo = 0xffffffffu;
        sh.hi = 0;
      }
      __syncthreads();
      {
        uint32_t lo = 0xffffffffu, hi = 0;
        each_logit<DT>(row, [&](float v, int) {
          if (bin_of(v) != b || !kept(v, weight(v, mx, q.inv_t))) return;
          lo = min(lo, ord_of(v));
          hi = max(hi, ord_of(v));
        });
        lo = ~wave_most(~lo);
        hi = wave_most(hi);
        if ((threadIdx.x & 63) == 0) {
          atomicMin(&sh.lo, lo);
          atomicMax(&sh.hi, hi);
        }
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
  if (equals > 0)
    last = nth_equal<DT>(a, row, cut, equals, sh);
  else if (equals == 0)
    last = (uint64_t)cut << 32;  // (cut 0: everything)

  // The draw: the blocks' kept weights first.
  auto keep = [&](float v, int i, double w) { return key_of(v, i) >= last && w >= q.min_p; };
  const int lane = threadIdx.x & 63;
  __syncthreads();
  for (int b = threadIdx.x >> 6; b < a.nb; b += kPickWaves) {
    float v[kUnit];
    load_unit<DT>(row, b * 64 + lane, v);
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      const double w = v[e] == kNegInf ? 0.0 : weight(v[e], mx, q.inv_t);
      if (v[e] != kNegInf && keep(v[e], (b * 64 + lane) * kUnit + e - row.lo, w)) s += w;
    }
    s = wave_sum(s);
    if (lane == 0) sh.l.w[b] = s;
  }
  draw_from_blocks<DT>(a, t, row, q, mx, sh, keep);
}

// The first largest logit.
template <int DT>
__device__ void pick_largest(const SampleArgs& a, int t, const Row& row, float mx,
                             PickShared& sh) {
  const int n = gather<DT>(a, row, mx, kMaxGroups, sh);  // the largest and its equals
  uint64_t best = 0;
  for (int i = threadIdx.x; i < min(n, kList); i += kPickThreads)
    best = best > sh.l.list[i] ? best : sh.l.list[i];
  if (n > kList) {  // (more equals than the list holds)
    each_logit<DT>(row, [&](float v, int i) {
      const uint64_t k = key_of(v, i);
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
    emit(a, t, index_of(best), 0.0);
  }
}

// The rest of a row whose list has at most 64 logits: filters (total: of all weights,
// where the list is only part of them; 0: the list's) and draw.  Wave w compares with
// the logits 8 w .. 8 w + 7, and wave 0 joins the parts.  Returns whether the list was
// enough.
__device__ bool pick_of_64(const SampleArgs& a, int t, const Params& q, float mx, int n,
                           double total, PickShared& sh) {
  static_assert(kPickWaves == 8, "eight logits to a wave");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool in = lane < n;
  uint64_t key = in ? sh.l.list[lane] : 0;
  int rank = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) rank += lane_of(key, wave * 8 + j) > key;
  int* ranks = (int*)sh.l.w;
  ranks[wave * 64 + lane] = rank;
  __syncthreads();
  rank = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) rank += ranks[w * 64 + lane];
  if (wave == 0 && in) sh.l.list[64 + rank] = key;
  __syncthreads();
  key = in ? sh.l.list[64 + lane] : 0;  // the lane's logit, larger ones before it
  const float v = logit_of(key);
  const double w = in ? weight(v, mx, q.inv_t) : 0.0;
  int m = q.min_p > 0.0 ? max(__builtin_popcountll(__ballot(in && w >= q.min_p)), 1) : n;
  if (q.k > 0) m = min(m, q.k);
  const double run = wave_upto(lane < m ? w : 0.0);
  if (q.p < 1.0) {
    const double sum = lane_of(run, m - 1), limit = q.p * (total > 0.0 ? total : sum);
    if (total > 0.0 && sum < limit) return false;
    const double before = dpp_from<0x138, 0xf>(run);
    m = max(__builtin_popcountll(__ballot(lane < m && before < limit)), 1);
  }
  const double all = lane_of(run, m - 1), target = q.u * all;
  // the kept weights up to the lane's logit, by index (added in the list's order)
  const int at = index_of(key);
  double part = 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int i = wave * 8 + j;
    const double wj = lane_of(w, i);
    part += i < m && __builtin_amdgcn_readlane(at, i) <= at ? wj : 0.0;
  }
  sh.l.w[512 + wave * 64 + lane] = part;
  __syncthreads();
  if (wave != 0) return true;
  double cum = 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) cum += sh.l.w[512 + j * 64 + lane];
  // the first by index that passes the target (none: the last of positive weight)
  const bool kept = lane < m && w > 0.0;
  const uint64_t pass = __ballot(kept && cum > target);
  // (indices are below 2^20; what is no candidate is 0)
  const uint32_t rate = !kept ? 0 : (!pass ? 1u + at : (cum > target ? (1u << 30) - at : 0));
  const uint32_t best = wave_most(rate);
  if (kept && rate == best) emit(a, t, at, log_prob(v, mx, q.inv_t, all));
  return true;
}

// A chain of dependent steps in one workgroup, whose latency bounds it (maxima, bound,
// groups, logits, sort, sums): 10 us for a row of top_k 50, 32 for 512 rows of all kinds.
template <int DT, bool DEFER>
__global__ __launch_bounds__(kPickThreads) __attribute__((amdgpu_waves_per_eu(4))) void pick_kernel(
    SampleArgs a) {
  __shared__ PickShared sh;
  const int t = blockIdx.x;
  const Row row = row_of<DT>(a, t);
  const Params q = params_of(a, t);
  if (DEFER && threadIdx.x == 0) a.open[t].state = 0;
  float mx = kNegInf;
  {
    constexpr int N = (kMaxGroups + kPickThreads - 1) / kPickThreads;
    float m[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = i * kPickThreads + threadIdx.x;
      m[i] = a.gmax[(size_t)t * a.ng + min(g, a.ng - 1)];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = i * kPickThreads + threadIdx.x;
      if (g < a.ng) sh.gmax[g] = m[i];
      mx = fmaxf(mx, m[i]);
    }
  }
  {
    const uint32_t o = wave_most(ord_of(mx));
    if ((threadIdx.x & 63) == 0) sh.parti[threadIdx.x >> 6] = (int)o;
    __syncthreads();
    uint32_t most = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) most = max(most, (uint32_t)sh.parti[w]);
    mx = of_ord(most);
  }
  if (mx == kNegInf) {  // no token
    if (threadIdx.x == 0) emit(a, t, -1, (double)kNegInf);
    return;
  }
  if (q.greedy) {
    pick_largest<DT>(a, t, row, mx, sh);
    return;
  }
  const bool all_in = a.V <= kList, bnd = bounded(a, q);
  if (q.k > 0 || q.p < 1.0 || q.min_p > 0.0) {
    float bound = kNegInf;
    double total = 0.0;  // of all weights, where top_p is the only filter
    if (bnd) {
      if (q.k > 0 && q.k <= min(a.ng, kMaxBound)) bound = bound_of(a, q.k, mx, sh);
      if (q.min_p > 0.0) {
        // a little below the logit of weight min_p
        const double v = (double)mx + log(q.min_p) / q.inv_t;
        bound = fmaxf(bound, (float)(v - fabs(v) * 1e-6 - 1e-30));
      }
    } else if (!all_in && q.k == 0) {
      double s = 0.0;
      for (int b = threadIdx.x; b < a.nb; b += kPickThreads) {
        const float ref = a.bref[(size_t)t * a.nb + b];
        s += ref == kNegInf ? 0.0 : a.bmass[(size_t)t * a.nb + b] * weight(ref, mx, q.inv_t);
      }
      total = block_sum(s, sh);
      bound = bound_of(a, min(a.ng, kTry), mx, sh);
    }
    const bool list = bnd || all_in || q.k == 0;  // (else a top_k beyond the bounds)
    // (rows that the launches after this one can take are left to them early)
    const int most = DEFER && q.k == 0 && !all_in ? kFewGroups : kMaxGroups;
    const int n = list ? gather<DT>(a, row, bound, most, sh) : kList + 1;
    if (n <= 64) {
      if (pick_of_64(a, t, q, mx, n, !bnd && !all_in ? total : 0.0, sh)) return;
    } else if (n <= kList) {
      sort_down(sh.l.list, n);
      int fit = 0;  // of at least min_p
      for (int i = threadIdx.x; i < n; i += kPickThreads) {
        const double w = weight(logit_of(sh.l.list[i]), mx, q.inv_t);
        sh.l.w[i] = w;
        fit += w >= q.min_p;
      }
      int m = q.min_p > 0.0 ? max(block_sum(fit, sh), 1) : n;
      if (q.k > 0) m = min(m, q.k);
      __syncthreads();
      bool done = true;
      if (q.p < 1.0) {
        running_sums(sh.l.w, m, sh);
        const double sum = sh.l.w[m - 1];
        // only top_p, and logits outside the list: the sum is that of the row
        const bool part = !bnd && !all_in;
        const double limit = q.p * (part ? total : sum);
        done = !part || sum >= limit;
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
    if constexpr (DEFER) {
      const bool by_bins = q.k == 0;
      if (by_bins)
        for (int i = threadIdx.x; i < kBins; i += kPickThreads)
          a.hist[(size_t)t * kBins + i] = 0;
      if (threadIdx.x == 0) {
        if (by_bins) a.open_rows[atomicAdd(a.open_n, 1)] = t;
        OpenRow o;
        o.state = by_bins ? 1 : 2;
        o.n = 0;
        o.mx = mx;
        o.bin = kBins;
        o.base = o.limit = 0.0;
        a.open[t] = o;
      }
    }
    return;
  }
  // no filter: the sums of the first launch
  __syncthreads();
  for (int b = threadIdx.x; b < a.nb; b += kPickThreads) {
    const float ref = a.bref[(size_t)t * a.nb + b];
    sh.l.w[b] = ref == kNegInf ? 0.0 : a.bmass[(size_t)t * a.nb + b] * weight(ref, mx, q.inv_t);
  }
  draw_from_blocks<DT>(a, t, row, q, mx, sh, [](float, int, double) { return true; });
}

// ---------------------------------------------------------------------------
// open rows: the bins' weights, the blocks' weights above the border, the cut
// ---------------------------------------------------------------------------

// The bin of a logit: 1/64 in log weight each, the last takes the rest.  (A bin that
// top_p is reached in is never the last: what lies below e^-31.9 of the largest weight
// is less than 2^20 e^-31.9, under the 2^-24 that a float top_p stays below 1.)
__device__ __forceinline__ int open_bin(double z) {
  const double x = z * -64.0;
  return x < (double)(kBins - 1) ? (int)x : kBins - 1;
}

// (Both kernels share the items, segments of open rows, among kOpenGrid workgroups.  A
// workgroup for each segment of every row would mostly find its row done: 512 rows of
// all kinds 20 and 39 us, 18 and 34 so.)
template <int DT, int BPW>
__global__ __launch_bounds__(kScanThreads) void hist_kernel(SampleArgs a, int segs) {
  __shared__ unsigned long long mass[kBins];
  const int items = *a.open_n * segs;
#pragma unroll 1
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int t = a.open_rows[item / segs], seg = item % segs;
    for (int i = threadIdx.x; i < kBins; i += kScanThreads) mass[i] = 0;
    const Row row = row_of<DT>(a, t);
    const Params q = params_of(a, t);
    if (q.p >= 1.0) continue;
    const float mx = a.open[t].mx;
    // log weights of at least min_p: all from `floor` on that weigh enough, all from
    // `floor_sure` on
    const double lnp = q.min_p > 0.0 ? log(q.min_p) : kLowest;
    const double floor = fmax(kLowest, lnp - 1e-9);
    const double floor_sure = q.min_p > 0.0 ? lnp + 1e-9 : kLowest;
    const int b0 = (seg * (kScanThreads / 64) + threadIdx.x / 64) * BPW;
    Raw<DT> raw[BPW];
    load_raws<DT, BPW>(row, b0 * 64, raw);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < BPW; ++i) {
      float u[kUnit];
      unpack<DT>(raw[0], u);
      next_raw(raw, raw[0]);
      int bin[kUnit];
      double w[kUnit];
      bool in[kUnit], rest = false;
#pragma unroll
      for (int e = 0; e < kUnit; ++e) {
        const double z = u[e] == mx ? 0.0 : z_of(u[e], mx, q.inv_t);
        in[e] = z >= floor;
        bin[e] = open_bin(z);
        rest |= in[e] && (bin[e] == kBins - 1 || z < floor_sure);
        // e^d, -1/64 < d <= 0, relative to the bin's top: the first term left
        // out, d^7 / 5040, is below 2^-54
        const double d = __builtin_fma((double)bin[e], 1.0 / 64.0, z);
        w[e] = 1.0 / 720;
        w[e] = __builtin_fma(w[e], d, 1.0 / 120);
        w[e] = __builtin_fma(w[e], d, 1.0 / 24);
        w[e] = __builtin_fma(w[e], d, 1.0 / 6);
        w[e] = __builtin_fma(w[e], d, 0.5);
        w[e] = __builtin_fma(w[e], d, 1.0);
        w[e] = __builtin_fma(w[e], d, 1.0);
      }
      if (__any(rest)) {  // the last bin, and weights next to min_p
#pragma unroll 1
        for (int e = 0; e < kUnit; ++e) {
          float v = u[0];
#pragma unroll
          for (int j = 1; j < kUnit; ++j) v = e == j ? u[j] : v;
          const double z = v == mx ? 0.0 : z_of(v, mx, q.inv_t);
          const bool ok = z >= floor && weight(v, mx, q.inv_t) >= q.min_p;
          const double far = weight_of(fmin(z + (kBins - 1) / 64.0, 0.0));
#pragma unroll
          for (int j = 0; j < kUnit; ++j)
            if (e == j) {
              in[j] = ok;
              if (bin[j] == kBins - 1) w[j] = far;
            }
        }
      }
#pragma unroll
      for (int e = 0; e < kUnit; ++e) {
        // (w 2^42 as the low bits of a float64 of that step)
        const long long fixed = __double_as_longlong(__builtin_fma(w[e], 0x1p42, 0x1p52)) & ((1ll << 52) - 1);
        if (in[e]) atomicAdd(&mass[bin[e]], (unsigned long long)fixed);
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kScanThreads)
      if (mass[i]) atomicAdd(&a.hist[(size_t)t * kBins + i], mass[i]);
    __syncthreads();
  }
}

template <int DT, int BPW>
__global__ __launch_bounds__(kScanThreads) void mark_kernel(SampleArgs a, int segs) {
  constexpr int W = kScanThreads / 64, PER = kBins / kScanThreads;
  __shared__ double part[W];
  __shared__ double running[kBins];
  __shared__ uint64_t mine[kList];  // the workgroup's logits of the border bin
  __shared__ int found, count, place;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int items = *a.open_n * segs;
#pragma unroll 1
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int t = a.open_rows[item / segs], seg = item % segs;
    __syncthreads();
    const Row row = row_of<DT>(a, t);
    const Params q = params_of(a, t);
    const float mx = a.open[t].mx;
    const double floor = kLowest;
    const int b0 = (seg * W + wave) * BPW;
    Raw<DT> raw[BPW];
    load_raws<DT, BPW>(row, b0 * 64, raw);
    // the border bin: every workgroup finds the same (without a top_p there is none)
    unsigned long long f[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) f[i] = a.hist[(size_t)t * kBins + threadIdx.x * PER + i];
    double m[PER], s = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) m[i] = (double)(q.p < 1.0 ? f[i] : 0) * 0x1p-42;
    {
      // (the bins' top weights: the first one's, then e^-1/64 apart)
      double w = weight_of(threadIdx.x * (-PER / 64.0));
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        m[i] *= w;
        w *= kBinStep;
        s += m[i];
      }
    }
    const double x = wave_upto(s);
    if (lane == 63) part[wave] = x;
    if (threadIdx.x == 0) {
      found = kBins;
      count = 0;
    }
    __syncthreads();
    double all = 0.0, run = x - s;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w < wave) run += part[w];
      all += part[w];
    }
    const double limit = q.p * all;
    // (the wave's first bin before the one atomic: 64 lanes' atomics on one word take
    // 2 us)
    uint32_t first = 0;  // its complement
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
      double r = run;
#pragma unroll
      for (int j = 0; j <= i; ++j) r += m[j];
      running[threadIdx.x * PER + i] = r;
      if (m[i] > 0.0 && r >= limit) first = ~(uint32_t)(threadIdx.x * PER + i);
    }
    first = wave_most(first);
    if (lane == 0 && first) atomicMin(&found, (int)~first);
    __syncthreads();
    const int border = found;
    if (seg == 0 && threadIdx.x == 0) {
      a.open[t].bin = border;
      a.open[t].limit = limit;
      a.open[t].base = border > 0 && border < kBins ? running[border - 1] : 0.0;
    }
    if (border == kBins && q.p < 1.0) continue;  // (rounding at the end: the row is done alone)
#pragma unroll 1
    for (int i = 0; i < BPW; ++i) {
      if (b0 + i >= a.nb) break;
      float u[kUnit];
      unpack<DT>(raw[0], u);
      next_raw(raw, raw[0]);
      double sum = 0.0;
      uint32_t listed = 0;
#pragma unroll
      for (int e = 0; e < kUnit; ++e) {
        const double z = u[e] == mx ? 0.0 : z_of(u[e], mx, q.inv_t);
        const double w = u[e] == mx ? 1.0 : weight_of(z);
        const int b = open_bin(z);
        const bool in = z >= floor && w >= q.min_p;
        sum += in && b < border ? w : 0.0;
        listed |= in && b == border ? 1u << e : 0u;
      }
      if (__any(listed)) {
        const int c = __builtin_popcount(listed), upto = wave_upto(c);
        int at = 0;
        if (lane == 63) at = atomicAdd(&count, upto);
        at = __builtin_amdgcn_readlane(at, 63) + upto - c;
#pragma unroll
        for (int e = 0; e < kUnit; ++e)
          if (listed >> e & 1) {
            if (at < kList) mine[at] = key_of(u[e], ((b0 + i) * 64 + lane) * kUnit + e - row.lo);
            ++at;
          }
      }
      sum = wave_sum(sum);
      if (lane == 0) a.bmass[(size_t)t * a.nb + b0 + i] = sum;
    }
    __syncthreads();
    if (threadIdx.x == 0 && count) place = atomicAdd(&a.open[t].n, count);
    __syncthreads();
    for (int i = threadIdx.x; i < min(count, kList); i += kScanThreads)
      if (place + i < kList) a.list[(size_t)t * kList + place + i] = mine[i];
  }
}

template <int DT>
__global__ __launch_bounds__(kPickThreads) __attribute__((amdgpu_waves_per_eu(4))) void finish_kernel(
    SampleArgs a) {
  const int t = blockIdx.x;
  const OpenRow o = a.open[t];
  if (o.state == 0) return;
  __shared__ PickShared sh;
  const Row row = row_of<DT>(a, t);
  const Params q = params_of(a, t);
  const bool border = q.p < 1.0;
  if (o.state == 2 || (border && (o.bin >= kBins - 1 || o.n > kList || o.limit <= 0.0))) {
    // (a function of its own takes its arguments from scratch: copies, so that nothing of
    // the kernel's lies there, whose rows mostly are done)
    const SampleArgs args = a;
    const Row alone = row;
    const Params par = q;
    whole_row<DT>(args, t, alone, par, o.mx, sh);
    return;
  }
  uint64_t last = 0;
  if (border) {
    for (int i = threadIdx.x; i < o.n; i += kPickThreads)
      sh.l.list[i] = a.list[(size_t)t * kList + i];
    last = last_of_list(o.n, o.base, o.limit, o.mx, q, sh);
  }
  // The border's kept logits join their blocks' sums, as whole numbers of 2^-42 of the
  // weight at the bin's top.
  unsigned long long* fixed = (unsigned long long*)sh.l.w;
  const double top = o.bin * (-1.0 / 64.0);
  __syncthreads();
  for (int b = threadIdx.x; b < a.nb; b += kPickThreads) fixed[b] = 0;
  __syncthreads();
  for (int i = threadIdx.x; border && i < o.n; i += kPickThreads) {
    const uint64_t k = sh.l.list[i];
    if (k < last) break;
    const float v = logit_of(k);
    const double z = v == o.mx ? 0.0 : z_of(v, o.mx, q.inv_t);
    atomicAdd(&fixed[(index_of(k) + row.lo) / kBlock],
              (unsigned long long)(weight_of(fmin(z - top, 0.0)) * 0x1p42));
  }
  __syncthreads();
  const double unit = border ? weight_of(top) * 0x1p-42 : 0.0;
  for (int b = threadIdx.x; b < a.nb; b += kPickThreads)
    sh.l.w[b] = a.bmass[(size_t)t * a.nb + b] + (double)fixed[b] * unit;
  draw_from_blocks<DT>(a, t, row, q, o.mx, sh,
                       [&](float v, int i, double w) { return key_of(v, i) >= last && w >= q.min_p; });
}

// The blocks of a scanned wave, and of a wave of the histograms' kernels in calls of few
// and of many blocks (rows of 150,000 logits, us with 2, 4: one scanned row 10.1, 11.9,
// 512 of them 91.0, 91.5; 16 open rows 72, 75, 32 91, 87, 128 167, 155).
constexpr int kScanBlocks = 2, kFewBlocks = 2, kManyBlocks = 4;
constexpr int kMany = 8192;
// Rows of one round of launches (the workspace is this many rows' at most).
constexpr int kRoundRows = 1024;

template <int DT>
hipError_t launch(SampleArgs a, hipStream_t stream) {
  constexpr int W = kScanThreads / 64;
  constexpr int ES = DT == PCTREE_F32 ? 4 : 2;
  const int rows = a.T;
  const bool filters = a.open && (a.has & (kHasTopP | kHasTopK | kHasMinP));
  for (int t0 = 0; t0 < rows; t0 += kRoundRows) {
    a.T = rows - t0 < kRoundRows ? rows - t0 : kRoundRows;
    const bool many = (long long)a.T * a.nb >= kMany;
    const int segs = (a.nb + W * kScanBlocks - 1) / (W * kScanBlocks);
    scan_kernel<DT, kScanBlocks><<<(unsigned)(a.T * segs), kScanThreads, 0, stream>>>(a, segs);
    if (filters) {
      pick_kernel<DT, true><<<(unsigned)a.T, kPickThreads, 0, stream>>>(a);
      // Rows are left to histograms by a top_p or min_p only.  (In every call that has one,
      // though its rows may all be settled, which then costs two empty launches: one row of
      // 150,000 logits with a top_k of 50 and a top_p takes 17.9 us in a graph, 16.1 without,
      // and 22.9 for 16.8 where the host issues them.  An open row takes 64, and 437 by one
      // workgroup.)
      if (a.has & (kHasTopP | kHasMinP)) {
        const int per = W * (many ? kManyBlocks : kFewBlocks);
        const int parts = (a.nb + per - 1) / per;
        const unsigned grid = (unsigned)std::min(a.T * parts, kOpenGrid);
        if (many) {
          hist_kernel<DT, kManyBlocks><<<grid, kScanThreads, 0, stream>>>(a, parts);
          mark_kernel<DT, kManyBlocks><<<grid, kScanThreads, 0, stream>>>(a, parts);
        } else {
          hist_kernel<DT, kFewBlocks><<<grid, kScanThreads, 0, stream>>>(a, parts);
          mark_kernel<DT, kFewBlocks><<<grid, kScanThreads, 0, stream>>>(a, parts);
        }
      }
      finish_kernel<DT><<<(unsigned)a.T, kPickThreads, 0, stream>>>(a);
    } else {
      pick_kernel<DT, false><<<(unsigned)a.T, kPickThreads, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.logits = (const char*)a.logits + (long long)a.T * a.row_stride * ES;
    a.uniform += a.T;
    a.temperature += a.T;
    a.top_k += a.T;
    a.top_p += a.T;
    a.min_p += a.T;
    a.token += a.T;
    if (a.logprob) a.logprob += a.T;
  }
  return hipSuccess;
}

}  // namespace

void plan_sample(int V, int* ng, int* nb, int* gshift) {
  const int span = V + kUnit - 1;  // elements from the 16-byte boundary on
  int s = 0;                       // (a group: the units of 1 << s lanes)
  while ((span + (kUnit << s) - 1) / (kUnit << s) > kMaxGroups - 1) ++s;
  *gshift = s;
  *ng = (span + (kUnit << s) - 1) / (kUnit << s);
  *nb = (span + kBlock - 1) / kBlock;
}

namespace {
int round_rows(int T) { return T < kRoundRows ? T : kRoundRows; }
bool deferring(int V) { return V > kList; }
}  // namespace

size_t sample_bytes(int T, int V) {
  int ng, nb, s;
  plan_sample(V, &ng, &nb, &s);
  size_t row = (size_t)nb * 12 + (size_t)ng * 4;
  if (deferring(V))
    row += (kBins + kList) * sizeof(uint64_t) + sizeof(OpenRow) + sizeof(int);
  return ((size_t)round_rows(T) * row + 16 + 511) / 256 * 256;
}

void place_sample(SampleArgs* a, void* workspace) {
  plan_sample(a->V, &a->ng, &a->nb, &a->gshift);
  const size_t T = (size_t)round_rows(a->T);
  char* w = (char*)workspace;
  a->hist = a->list = nullptr;
  a->open = nullptr;
  a->open_n = a->open_rows = nullptr;
  if (deferring(a->V)) {
    a->hist = (unsigned long long*)w;
    a->list = a->hist + T * kBins;
    a->open = (OpenRow*)(a->list + T * kList);
    w = (char*)(a->open + T);
  }
  a->bmass = (double*)w;
  a->bref = (float*)(a->bmass + T * a->nb);
  a->gmax = a->bref + T * a->nb;
  if (a->open) {
    a->open_n = (int*)(a->gmax + T * a->ng);
    a->open_rows = a->open_n + 1;
  }
}

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PCTREE_F32: return launch<PCTREE_F32>(a, stream);
    case PCTREE_BF16: return launch<PCTREE_BF16>(a, stream);
    default: return launch<PCTREE_F16>(a, stream);
  }
}

}  // namespace pctree
