// Penalties for repeated tokens, biases and a grammar's mask on rows of logits, in place.
//
// forbid_kernel: -inf where a row's mask has no bit, eight logits to a lane; eight that are
// all forbidden are written without being read.  A line of 128 bytes is written whole where
// any of its logits is forbidden, its groups without one read and written back, and not
// touched where none is.  Waves wait for most of their time (142 of 181 million wave clocks
// in the call below): each does one piece, whose row, words, logits and stores follow one
// another.
// adjust_kernel: a workgroup takes a segment of the vocabulary and some rows of one
// request.  It counts the request's history in a table of the segment in LDS, so a token's
// count costs no memory beside the history itself, whatever the history's length; then
// each wave goes over rows by itself, or over its share of the tokens where rows are few,
// and touches only the tokens that the table holds.  A tree's node counts its ancestors'
// tokens: those in the segment are few, and listed for each row.  One row after 2000
// tokens 5.4 us: parameters, history, table and logits in a chain; 512 rows of four trees
// 22 us, their tokens' lines of memory.  64 single rows of 151,936 after 4000 tokens each 21
// us, of which 13 are 4800 workgroups that clear and search a table each (as long after 4
// tokens), 5 their reading the history, 75 times a request, and 3 the lines.  (A table that
// holds most of a small vocabulary: 512 rows of 1,827 tokens 70 us with waves by rows
// alone, 14 so.)
// (Segments of 4096 tokens took 124 us for the 512 rows where these take 84, a mask's pass
// in this kernel included at the time: fewer workgroups fit a compute unit; of 1024, 106.)
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "pctree_step.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSegment = 2048;  // tokens of a workgroup
constexpr int kLine = 128;      // bytes that memory writes without reading them first
constexpr int kBatch = 8;       // tokens of the history that a thread loads together
constexpr int kRows = 4;        // rows that a wave of adjust_kernel has in flight
constexpr int kSteps = 4;       // groups of eight logits that a lane of forbid_kernel does
// a token's entry of the table
constexpr uint32_t kSeen = 1u << 31;     // in the prompt
constexpr uint32_t kBias = 1u << 30;     // has a bias
constexpr uint32_t kNode = 1u << 29;     // a tree node's token
constexpr uint32_t kCount = kNode - 1u;  // how often among the tokens after the prompt

// Eight logits, from a 16-byte boundary.
template <typename T>
struct Eight {  // (of 16 bits)
  u32x4 w;
  __device__ __forceinline__ void load(const T* p) {
    w = __builtin_nontemporal_load((const u32x4*)p);
  }
  __device__ __forceinline__ void store(T* p) const {
    __builtin_nontemporal_store(w, (u32x4*)p);
  }
  // -inf where a bit is set
  __device__ __forceinline__ void forbid(uint32_t no) {
    constexpr uint32_t inf = (uint32_t)__builtin_bit_cast(uint16_t, (T)kNegInf) * 0x10001u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = (uint32_t)((int)(no << (31 - 2 * e)) >> 31);
      const uint32_t hi = (uint32_t)((int)(no << (30 - 2 * e)) >> 31);
      const uint32_t m = (lo & 0xffffu) | (hi & 0xffff0000u);
      w[e] = (inf & m) | (w[e] & ~m);
    }
  }
};
template <>
struct Eight<float> {
  f32x4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = __builtin_nontemporal_load((const f32x4*)p);
    w[1] = __builtin_nontemporal_load((const f32x4*)(p + 4));
  }
  __device__ __forceinline__ void store(float* p) const {
    __builtin_nontemporal_store(w[0], (f32x4*)p);
    __builtin_nontemporal_store(w[1], (f32x4*)(p + 4));
  }
  __device__ __forceinline__ void forbid(uint32_t no) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if ((no >> e) & 1u) w[e / 4][e % 4] = kNegInf;
  }
};

// Request r's rows, clamped as the interface says.
struct Rows {
  int start, cnt;
};
__device__ __forceinline__ Rows rows_of(const AdjustArgs& a, int start, int cnt) {
  cnt = start >= 0 && start < a.T ? min(min(max(cnt, 0), a.max_rows), a.T - start) : 0;
  return {start, a.token ? min(cnt, a.N) : cnt};
}

// Waves of a row (one starts up to a line before it).
__host__ int row_parts(int V) { return (V + kLine + kSteps * 512 - 1) / (kSteps * 512); }

// A wave takes kSteps * 512 logits of a row.  512 rows of 151936 bfloat16 with masks of
// 0.1 to 90 % of the tokens, 186 MB read and written: 43 us, 4.3 TB/s (53 with stores of
// the groups that change alone, and the cache's ordinary policy).
template <typename T>
__global__ __launch_bounds__(kThreads) void forbid_kernel(AdjustArgs a, int parts) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + threadIdx.x / 64);
  const int t = wave / parts, part = wave % parts;
  if (t >= a.T) return;
  const int m = a.allowed_row ? a.allowed_row[t] : t;
  if ((unsigned)m >= (unsigned)a.M) return;
  bool ours = false;  // (a request's row)
  for (int r0 = 0; r0 < a.R && !ours; r0 += 64) {
    const int r = min(r0 + lane, a.R - 1);
    const Rows q = rows_of(a, a.row_start[r], a.row_count[r]);
    ours = __any(t >= q.start && t - q.start < q.cnt);
  }
  if (!ours) return;
  T* row = (T*)a.logits + t * a.row_stride;
  const uint32_t* words = a.allowed + (size_t)m * a.AW;
  // groups of eight from the line's start before the row: `shift` logits of the first lie
  // before it
  const int shift = (int)(((uintptr_t)row & (kLine - 1)) / sizeof(T));
  const int first = part * kSteps * 512 + lane * 8 - shift;
  uint32_t no[kSteps];  // forbidden
  bool whole[kSteps];
  Eight<T> x[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int at = first + s * 512, w = at >> 5;  // (floor)
    uint64_t ok = words[min(max(w, 0), a.AW - 1)];
    if (shift) ok |= (uint64_t)words[min(max(w + 1, 0), a.AW - 1)] << 32;
    // (of the eight, those of the row)
    const uint32_t inside = at >= a.V || at <= -8 ? 0u
                            : (0xffu >> max(at + 8 - a.V, 0)) & (0xffu << max(-at, 0));
    no[s] = ~(uint32_t)(ok >> (at & 31)) & inside;
    // a line is written whole or not at all
    constexpr int per = kLine / (8 * sizeof(T));
    const uint64_t line = (__ballot(no[s] != 0) >> (lane / per * per)) & ((1ull << per) - 1);
    whole[s] = inside == 0xffu && line;
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    x[s] = {};
    if (whole[s] && no[s] != 0xffu) x[s].load(row + first + s * 512);
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int at = first + s * 512;
    if (whole[s]) {
      x[s].forbid(no[s]);
      x[s].store(row + at);
    } else {  // (beside another row's logits)
      for (uint32_t todo = no[s]; todo; todo &= todo - 1) row[at + __builtin_ctz(todo)] = (T)kNegInf;
    }
  }
}

struct Penalty {
  float repetition, frequency, presence;
};

// The logit of a token that is there `count` times after the prompt.
__device__ __forceinline__ float penalised(float x, bool seen, uint32_t count, const Penalty& p) {
  if (seen) x = x > 0.0f ? x / p.repetition : x * p.repetition;
  if (count) x = x - p.frequency * (float)count - p.presence;
  return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a, int segments, int groups) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  uint32_t* table = lds;                                               // [kSegment]
  uint32_t* bias = table + kSegment;                                   // [kSegment] where there are biases
  uint16_t* list = (uint16_t*)(bias + (a.bias_token ? kSegment : 0));  // [kSegment] tokens in the table
  uint16_t* node_at = list + kSegment;                                 // [N] tree tokens in the segment
  uint16_t* node_is = node_at + (a.token ? a.N : 0);                   // [N] and their nodes
  __shared__ int sListed, sNodes;

  const int seg = blockIdx.x % segments, rg = blockIdx.x / segments;
  const int r = rg / groups, group = rg % groups;
  // (read together, what is not given as something that is)
  const auto at = [r](const auto* p, const void* other) { return p ? p[r] : ((decltype(p))other)[r]; };
  const int start = a.row_start[r], row_count = a.row_count[r];
  const int h_start = at(a.history_start, a.row_start), h_count = at(a.history_count, a.row_start);
  const int h_prompt = at(a.prompt_count, a.row_start);
  const int b_start = at(a.bias_start, a.row_start), b_count = at(a.bias_count, a.row_start);
  Penalty p = {at(a.repetition, a.row_start), at(a.frequency, a.row_start), at(a.presence, a.row_start)};
  if (!a.repetition || !(p.repetition > 0.0f) || p.repetition == __builtin_inff()) p.repetition = 1.0f;
  if (!a.frequency || !(fabsf(p.frequency) < __builtin_inff())) p.frequency = 0.0f;
  if (!a.presence || !(fabsf(p.presence) < __builtin_inff())) p.presence = 0.0f;
  const bool penalties = p.repetition != 1.0f || p.frequency != 0.0f || p.presence != 0.0f;
  const int cnt = rows_of(a, start, row_count).cnt;
  const int per = (cnt + groups - 1) / groups;  // (of the rows there are)
  const int first = group * per, last = min(first + per, cnt);
  if (first >= last) return;
  const int v0 = seg * kSegment, width = min(kSegment, a.V - v0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;

  if (threadIdx.x == 0) sListed = sNodes = 0;
  for (int i = threadIdx.x * 4; i < kSegment; i += kThreads * 4) {
    *(u32x4*)(table + i) = u32x4{0u, 0u, 0u, 0u};
    if (a.bias_token) *(u32x4*)(bias + i) = u32x4{0u, 0u, 0u, 0u};
  }
  __syncthreads();
  if (penalties && a.history) {
    const int h0 = min(max(h_start, 0), a.history_total);
    const int hn = min(max(h_count, 0), a.history_total - h0);
    const int pn = a.prompt_count ? min(max(h_prompt, 0), hn) : 0;
    for (int i0 = threadIdx.x; i0 < hn; i0 += kBatch * kThreads) {
      uint32_t at[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        at[k] = (uint32_t)a.history[h0 + min(i0 + k * kThreads, hn - 1)] - (uint32_t)v0;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = i0 + k * kThreads;
        if (i >= hn || at[k] >= (uint32_t)width) continue;
        if (i < pn) atomicOr(&table[at[k]], kSeen);
        else atomicAdd(&table[at[k]], 1u);
      }
    }
  }
  if (a.bias_token) {  // the last of a token's entries holds
    const int b0 = min(max(b_start, 0), a.bias_total);
    const int bn = min(max(b_count, 0), a.bias_total - b0);
    for (int i = threadIdx.x; i < bn; i += kThreads) {
      const uint32_t at = (uint32_t)a.bias_token[b0 + i] - (uint32_t)v0;
      if (at >= (uint32_t)width) continue;
      atomicMax(&bias[at], (uint32_t)(b0 + i) + 1u);
      atomicOr(&table[at], kBias);
    }
  }
  if (penalties && a.token) {
    for (int j = threadIdx.x; j < cnt; j += kThreads) {
      const uint32_t at = (uint32_t)a.token[(size_t)r * a.N + j] - (uint32_t)v0;
      if (at >= (uint32_t)width) continue;
      atomicOr(&table[at], kNode);
      const int k = atomicAdd(&sNodes, 1);
      node_at[k] = (uint16_t)at;
      node_is[k] = (uint16_t)j;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kSegment; i += kThreads) {  // (a wave: 64 tokens in turn)
    const bool there = table[i] != 0;
    const uint64_t all = __ballot(there);
    int first = 0;
    if (all && lane == 0) first = atomicAdd(&sListed, __builtin_popcountll(all));
    first = __builtin_amdgcn_readfirstlane(first);
    if (there) list[first + __builtin_popcountll(all & ((1ull << lane) - 1))] = (uint16_t)i;
  }
  __syncthreads();
  const int listed = sListed, nodes = sNodes;

  // Rows of a wave a few at a time, whose loads all issue before the first is used; 64 of
  // the table's tokens, one to a lane.  Where the workgroup has few rows its waves share
  // them and take tokens in turn.
  const int rows = last - first;
  const bool share = rows <= kRows;
  const int apart = share ? 1 : kWaves;  // rows of a wave
  const int k_first = share ? wave * 64 : 0, k_step = share ? kWaves * 64 : 64;
  const auto adjust = [&](auto number, int i0) {
    constexpr int K = number.value;
    int i[K], m[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      i[j] = min(i0 + j * apart, last - 1);
      m[j] = !a.allowed ? -1 : a.allowed_row ? a.allowed_row[start + i[j]] : start + i[j];
    }
    for (int k0 = k_first; k0 < listed; k0 += k_step) {
      const bool has = k0 + lane < listed;
      const int at = list[min(k0 + lane, listed - 1)];
      const uint32_t e = table[at];
      const float b = e & kBias ? a.bias_value[bias[at] - 1u] : 0.0f;
      T* place[K];
      T x[K];
      uint32_t ok[K], n[K];
#pragma unroll
      for (int j = 0; j < K; ++j) {
        place[j] = (T*)a.logits + (long long)(start + i[j]) * a.row_stride + v0 + at;
        x[j] = *place[j];
        n[j] = e & kCount;
        ok[j] = ~0u;
        if ((unsigned)m[j] < (unsigned)a.M) ok[j] = a.allowed[(size_t)m[j] * a.AW + ((v0 + at) >> 5)];
      }
      // and how often it is among the row's node and its ancestors
      for (int l0 = 0; l0 < nodes; l0 += 64) {
        const int l = min(l0 + lane, nodes - 1), node = node_is[l], token = node_at[l];
        uint32_t word[K];
#pragma unroll
        for (int j = 0; j < K; ++j) word[j] = a.mask[((size_t)r * a.N + i[j]) * a.NW + (node >> 5)];
#pragma unroll
        for (int j = 0; j < K; ++j) {
          if (i0 + j * apart >= last) break;
          uint64_t in = __ballot(l0 + lane < nodes && ((word[j] >> (node & 31)) & 1u));
          for (; in; in &= in - 1)
            n[j] += __builtin_amdgcn_readlane(token, (int)__builtin_ctzll(in)) == at;
        }
      }
#pragma unroll
      for (int j = 0; j < K; ++j) {
        const bool seen = (e & kSeen) || n[j];
        float y = penalised((float)x[j], seen, n[j], p);
        if (e & kBias) y += b;
        if (has && (seen || (e & kBias)) && i0 + j * apart < last && ((ok[j] >> (at & 31)) & 1u))
          *place[j] = (T)y;
      }
    }
  };
  if (rows == 1) {
    adjust(std::integral_constant<int, 1>{}, first);
  } else {
    for (int i0 = share ? first : first + wave; i0 < last; i0 += kRows * apart)
      adjust(std::integral_constant<int, kRows>{}, i0);
  }
}

// Groups of a request's rows: of kRows at least, fewer where they leave compute units idle
// (64 nodes over 3,831 tokens 9.4 us with four rows, 6.8 with one; over 32,000 with one
// 8.4, with four 7.1).
int row_groups(const AdjustArgs& a, int segments) {
  const long long pairs = (long long)a.R * segments;
  const auto groups = [&](int blocks, int most) {
    return std::min<long long>((blocks + pairs - 1) / pairs, most);
  };
  return (int)std::max({1ll, groups(1024, a.max_rows / kRows), groups(256, a.max_rows)});
}

template <typename T>
hipError_t launch(const AdjustArgs& a, hipStream_t stream) {
  if (a.allowed) {
    const int parts = row_parts(a.V);
    const long long waves = (long long)a.T * parts;
    forbid_kernel<T><<<(unsigned)((waves + kWaves - 1) / kWaves), kThreads, 0, stream>>>(a, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const bool penalties = (a.repetition || a.frequency || a.presence) && (a.history || a.token);
  if (!penalties && !a.bias_token) return hipSuccess;
  const int segments = (a.V + kSegment - 1) / kSegment, groups = row_groups(a, segments);
  const unsigned blocks = (unsigned)((long long)a.R * segments * groups);
  const unsigned lds = kSegment * (4 + (a.bias_token ? 4 : 0) + 2) + (a.token ? 4 * a.N : 0);
  adjust_kernel<T><<<blocks, kThreads, lds, stream>>>(a, segments, groups);
  return hipGetLastError();
}

}  // namespace

bool adjust_fits(const AdjustArgs& a) {
  const long long parts = row_parts(a.V);
  return (long long)a.T * parts <= INT32_MAX - kThreads &&
         ((long long)a.T * parts + kWaves - 1) / kWaves <= (1 << 24) - 1 &&
         (long long)a.R * ((a.V + kSegment - 1) / kSegment) + 1024 <= (1 << 24) - 1;
}

hipError_t launch_adjust(const AdjustArgs& a, int dtype, hipStream_t stream) {
  if (dtype == PCTREE_F32) return launch<float>(a, stream);
  if (dtype == PCTREE_BF16) return launch<__bf16>(a, stream);
  return launch<_Float16>(a, stream);
}

}  // namespace pctree
