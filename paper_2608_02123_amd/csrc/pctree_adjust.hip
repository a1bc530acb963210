// Penalties for repeated tokens, biases and a grammar's mask on rows of logits, in place.
//
// A workgroup takes a segment of the vocabulary and some rows of one request.  It counts
// the request's history in a table of the segment in LDS, so a token's count costs no
// memory beside the history itself, whatever the history's length; then each wave goes
// over rows by itself.  A row without a mask is touched only at the tokens that the table
// holds; a row with one is written where the mask forbids, without being read where it
// forbids eight tokens in a row.  A tree's node counts its ancestors' tokens: those in the
// segment are listed, few, and looked at for each row.
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pctree_step.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSegment = 4096;  // tokens of a workgroup
// a token's entry of the table
constexpr uint32_t kSeen = 1u << 31;     // in the prompt
constexpr uint32_t kBias = 1u << 30;     // has a bias
constexpr uint32_t kNode = 1u << 29;     // a tree node's token
constexpr uint32_t kCount = kNode - 1u;  // how often among the tokens after the prompt

struct Penalty {
  float repetition, frequency, presence;
};

__device__ __forceinline__ float finite_or(float x, float other) {
  return fabsf(x) < __builtin_inff() ? x : other;
}

// The logit of a token that is there `count` times after the prompt.
__device__ __forceinline__ float penalised(float x, bool seen, uint32_t count, const Penalty& p) {
  if (seen) x = x > 0.0f ? x / p.repetition : x * p.repetition;
  if (count) x = x - p.frequency * (float)count - p.presence;
  return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a, int segments, int groups) {
  extern __shared__ uint32_t lds[];
  uint32_t* table = lds;                                          // [kSegment]
  uint32_t* bias = table + kSegment;                              // [kSegment] where there are biases
  uint16_t* list = (uint16_t*)(bias + (a.bias_token ? kSegment : 0));  // [kSegment] tokens in the table
  uint16_t* node_at = list + kSegment;                            // [N] tree tokens in the segment
  uint16_t* node_is = node_at + (a.token ? a.N : 0);              // [N] and their nodes
  __shared__ int sListed, sNodes;

  const int seg = blockIdx.x % segments, rg = blockIdx.x / segments;
  const int r = rg / groups, group = rg % groups;
  const int start = a.row_start[r];
  int cnt = start >= 0 && start < a.T ? min(min(max(a.row_count[r], 0), a.max_rows), a.T - start) : 0;
  if (a.token) cnt = min(cnt, a.N);
  const int per = (a.max_rows + groups - 1) / groups;
  const int first = group * per, last = min(first + per, cnt);
  if (first >= last) return;
  const int v0 = seg * kSegment, width = min(kSegment, a.V - v0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;

  Penalty p = {1.0f, 0.0f, 0.0f};
  if (a.repetition) p.repetition = finite_or(a.repetition[r], 1.0f);
  if (!(p.repetition > 0.0f)) p.repetition = 1.0f;
  if (a.frequency) p.frequency = finite_or(a.frequency[r], 0.0f);
  if (a.presence) p.presence = finite_or(a.presence[r], 0.0f);
  const bool penalties = p.repetition != 1.0f || p.frequency != 0.0f || p.presence != 0.0f;

  if (threadIdx.x == 0) sListed = sNodes = 0;
  for (int i = threadIdx.x; i < kSegment; i += kThreads) {
    table[i] = 0;
    if (a.bias_token) bias[i] = 0;
  }
  __syncthreads();
  if (penalties && a.history) {
    const int h0 = min(max(a.history_start[r], 0), a.history_total);
    const int hn = min(max(a.history_count[r], 0), a.history_total - h0);
    const int pn = a.prompt_count ? min(max(a.prompt_count[r], 0), hn) : 0;
    for (int i = threadIdx.x; i < hn; i += kThreads) {
      const uint32_t at = (uint32_t)a.history[h0 + i] - (uint32_t)v0;
      if (at >= (uint32_t)width) continue;
      if (i < pn) atomicOr(&table[at], kSeen);
      else atomicAdd(&table[at], 1u);
    }
  }
  if (a.bias_token) {  // the last of a token's entries holds
    const int b0 = min(max(a.bias_start[r], 0), a.bias_total);
    const int bn = min(max(a.bias_count[r], 0), a.bias_total - b0);
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
  for (int i = threadIdx.x; i < width; i += kThreads)
    if (table[i]) list[atomicAdd(&sListed, 1)] = (uint16_t)i;
  __syncthreads();
  const int listed = sListed, nodes = sNodes;

  for (int i = first + wave; i < last; i += kWaves) {
    const long long t = start + i;
    T* row = (T*)a.logits + t * a.row_stride + v0;
    const uint32_t* words = a.token ? a.mask + ((size_t)r * a.N + i) * a.NW : nullptr;
    // how often token `at` is among the row's node and its ancestors
    const auto above = [&](int at) {
      uint32_t n = 0;
      for (int k0 = 0; k0 < nodes; k0 += 64) {
        const int k = min(k0 + lane, nodes - 1), j = node_is[k];
        uint64_t in = __ballot(k0 + lane < nodes && ((words[j >> 5] >> (j & 31)) & 1u));
        const int mine = node_at[k];
        while (in) {
          const int l = (int)__builtin_ctzll(in);
          in &= in - 1;
          n += __builtin_amdgcn_readlane(mine, l) == at;
        }
      }
      return n;
    };
    const auto settled = [&](float x, int at, uint32_t e, uint32_t n) {
      n += e & kCount;
      x = penalised(x, (e & kSeen) || n, n, p);
      if (e & kBias) x += a.bias_value[bias[at] - 1u];
      return x;
    };
    int m = -1;
    if (a.allowed) {
      m = a.allowed_row ? a.allowed_row[t] : (int)t;
      if ((unsigned)m >= (unsigned)a.M) m = -1;
    }
    if (m < 0) {
      for (int k0 = 0; k0 < listed; k0 += 64) {
        const int at = list[min(k0 + lane, listed - 1)];
        const uint32_t n = above(at);
        if (k0 + lane < listed) {
          const uint32_t e = table[at];
          const float x = (float)row[at];
          row[at] = (T)settled(x, at, e, n);
        }
      }
      continue;
    }
    const uint8_t* bits = (const uint8_t*)(a.allowed + (size_t)m * a.AW) + v0 / 8;
    for (int b0 = 0; b0 < width; b0 += 512) {
      const int at = b0 + lane * 8;
      const int n8 = min(max(width - at, 0), 8);
      const uint32_t ok = n8 > 0 ? bits[at / 8] : 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t entry = e < n8 ? table[at + e] : 0u;
        const uint32_t n = nodes ? above(at + e) : 0u;
        if (e < n8) {
          if (!((ok >> e) & 1u)) row[at + e] = (T)kNegInf;
          else if (entry) row[at + e] = (T)settled((float)row[at + e], at + e, entry, n);
        }
      }
    }
  }
}

int row_groups(const AdjustArgs& a, int segments) {
  const long long pairs = (long long)a.R * segments;
  const long long want = (1024 + pairs - 1) / pairs, most = (a.max_rows + kWaves - 1) / kWaves;
  return (int)std::max(1ll, std::min(want, most));
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& a, int dtype, hipStream_t stream) {
  const int segments = (a.V + kSegment - 1) / kSegment, groups = row_groups(a, segments);
  const unsigned blocks = (unsigned)((long long)a.R * segments * groups);
  const unsigned lds = kSegment * (4 + (a.bias_token ? 4 : 0) + 2) + (a.token ? 4 * a.N : 0);
  if (dtype == PCTREE_F32) adjust_kernel<float><<<blocks, kThreads, lds, stream>>>(a, segments, groups);
  else if (dtype == PCTREE_BF16) adjust_kernel<__bf16><<<blocks, kThreads, lds, stream>>>(a, segments, groups);
  else adjust_kernel<_Float16><<<blocks, kThreads, lds, stream>>>(a, segments, groups);
  return hipGetLastError();
}

}  // namespace pctree
