// A paged cache in 8 bits (pctree_held.h): new rows into their pages, and compaction
// after acceptance.  A block of slots of one head has one scale, so a block, not a row,
// is what a wave writes.
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pctree_held.h"
#include "pctree_paged.h"
#include "pctree_rows.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

constexpr int kQueries = 4;  // loads that a wave of queries has in flight

// The queries of row t: `part` of `split` waves, 512 / D heads at a time.
template <int D, bool H>
__device__ __forceinline__ void append_queries(const AppendArgs& a, int t, int part, int split) {
  constexpr int LPH = D / 8, HPW = 64 / LPH;
  const int lane = threadIdx.x & 63, e0 = (lane % LPH) * 8;
  const int r = request_of_row(a.b, t);
  if (r < 0) return;
  const PagedReq rq = paged_req(a.b, r);
  const bool turns = a.rope && e0 < a.rot;
  Turn turn;
  if (turns) load_turn(a, a.position ? a.position[t] : rq.prefix + (t - rq.start), e0, turn);
  for (int i0 = part * HPW; i0 < a.Hq; i0 += kQueries * split * HPW) {
    u32x4 x[kQueries];
#pragma unroll
    for (int k = 0; k < kQueries; ++k) {  // (heads past the last: it again)
      const int h = min(i0 + k * split * HPW + lane / LPH, a.Hq - 1);
      x[k] = *(const u32x4*)(a.q + t * a.q_stride + h * D + e0);
    }
#pragma unroll
    for (int k = 0; k < kQueries; ++k) {
      const int h = i0 + k * split * HPW + lane / LPH;
      if (i0 + k * split * HPW >= a.Hq) break;
      float y[8];
      unpack8<H>(x[k], y);
      if (a.q_norm) norm_head<D, H>(y, a.q_norm, a.eps, e0);
      if (a.rope) turn_head<D>(a, y, turn, e0, turns);
      if (h < a.Hq) *(u32x4*)(a.q_out + t * a.q_out_stride + h * D + e0) = pack8<H>(y);
    }
  }
}

// How the waves of a workgroup share blocks of G slots of one head: `waves` of them to a
// block, `steps` loads of 512 / D rows each.  (A wave by itself took 31 us for the keys and
// values of 8000 rows in blocks of 32, and the registers of eight steps left three waves a
// SIMD.)
template <int D, int G>
struct Share {
  static constexpr int rows = 512 / D;
  static constexpr int waves = G / rows < kWaves ? G / rows : kWaves;
  static constexpr int steps = G / rows / waves;
  static constexpr int heads = kWaves / waves;
};

// The n new rows t .. of a block of G slots, the first at offset o0 (slots below it hold
// rows from before), of one head of the keys or the values, by wave `part` of those that
// share it: the rows stay in registers between their largest magnitude, which the waves
// join in `most`, and their rounding.  Without `live` the wave only keeps the others'
// company at the barrier.
template <int D, bool H, int G>
__device__ __forceinline__ void append_block(const AppendArgs& a, bool live, bool keys, int h, int t,
                                             int n, int o0, int slot0, uint8_t* block,
                                             uint8_t* scale, int part, float* most) {
  using S = Share<D, G>;
  constexpr int LPH = D / 8;
  const int lane = threadIdx.x & 63, e0 = (lane % LPH) * 8;
  const int j0 = part * S::steps * S::rows + lane / LPH;  // the lane's first slot of the block
  const bool any = live && j0 - lane / LPH < o0 + n && j0 - lane / LPH + S::steps * S::rows > o0;
  const bool turns = keys && a.rope && e0 < a.rot;
  float y[S::steps][8];
  int was = 0;
  float large = 0.0f;
  if (any) {  // (the same in every lane; lanes beside the rows repeat one of them)
    const uint16_t* src = (keys ? a.k : a.v) + h * D + e0;
    const long long stride = keys ? a.k_stride : a.v_stride;
    u32x4 x[S::steps];
    int pos[S::steps];
#pragma unroll
    for (int s = 0; s < S::steps; ++s) {
      const int i = min(max(j0 + s * S::rows - o0, 0), n - 1);
      x[s] = *(const u32x4*)(src + (t + i) * stride);
      pos[s] = turns && a.position ? a.position[t + i] : slot0 + i;
    }
#pragma unroll
    for (int s = 0; s < S::steps; ++s) {
      Turn turn;
      if (turns) load_turn(a, pos[s], e0, turn);
      unpack8<H>(x[s], y[s]);
      if (keys && a.k_norm) norm_head<D, H>(y[s], a.k_norm, a.eps, e0);
      if (keys && a.rope) turn_head<D>(a, y[s], turn, e0, turns);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = fabsf(y[s][e]);
        large = m < __builtin_inff() ? fmaxf(large, m) : large;
      }
    }
    large = wave_max(large);
  }
  if (live && o0 > 0) was = scale_in(*scale);
  if constexpr (S::waves > 1) {
    const int first = threadIdx.x / 64 - part;
    if (lane == 0) most[first + part] = large;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < S::waves; ++w) large = fmaxf(large, most[first + w]);
  }
  if (!live) return;
  const int now = max(scale_of(large), was);
  if (any) {
    const float down = scale_down(now);
#pragma unroll
    for (int s = 0; s < S::steps; ++s) {
      const int j = j0 + s * S::rows;
      if (j < o0 || j >= o0 + n) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[s][e] *= down;
      *(uint2*)(block + j * D + e0) = hold8(y[s]);
    }
  }
  if (now == was) return;
  const float f = scale_up(127 - min(now - was, 126));
  for (int j = part * S::rows + lane / LPH; j < o0; j += S::waves * S::rows) {
    uint2* p = (uint2*)(block + j * D + e0);  // the rows from before under the grown scale
    uint2 w = *p;
    w.x = rescale4(w.x, f);
    w.y = rescale4(w.y, f);
    *p = w;
  }
  if (part == 0 && lane == 0) *scale = (uint8_t)now;
}

// Workgroups of keys and values first, whose chains are long: each takes, of `window`
// rows, the blocks whose first new row is among these, for Share's heads of the keys or the
// values, or (Both) of the keys and then the values.  Then qblocks of queries, qsplit waves
// a row.  Bytes bound them (7900 rows of 32 and 8 heads of 128, 182 MB: 45 us, 4.0 TB/s).
template <int D, bool H, int G, bool Both>
__global__ __launch_bounds__(kThreads) void append8_kernel(AppendArgs a, HeldScales sc, int qblocks,
                                                          int qsplit, int window) {
  using S = Share<D, G>;
  __shared__ float most[2][kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int kvblocks = gridDim.x - qblocks;
  if ((int)blockIdx.x >= kvblocks) {
    const int w = (blockIdx.x - kvblocks) * kWaves + wave;
    if (w / qsplit < a.b.T) append_queries<D, H>(a, w / qsplit, w % qsplit, qsplit);
    return;
  }
  const int items = Both ? a.Hkv : 2 * a.Hkv;
  const int groups = (items + S::heads - 1) / S::heads;  // of heads
  const int b = blockIdx.x;
  const int item = b % groups * S::heads + wave / S::waves, h = item % a.Hkv;
  const bool live = item < items;
  const int t0 = b / groups * window, end = min(t0 + window, a.b.T);
  const int blocks = 1 << (a.b.page_shift - sc.block_shift);  // of a page
  int turn = 0;
  for (int t = t0; t < end;) {  // (the same in every wave)
    const int r = request_of_row(a.b, t);
    if (r < 0) {
      ++t;
      continue;
    }
    const PagedReq rq = paged_req(a.b, r);
    const int i = t - rq.start, slot = rq.prefix + i, o0 = slot % G;
    const int n = min(G - o0, rq.cnt - i);  // rows to the block's end
    if (i == 0 || o0 == 0) {
      const int page =
          slot < a.b.C ? a.b.page_table[(size_t)r * a.b.max_pages + (slot >> a.b.page_shift)] : -1;
      if ((unsigned)page < (unsigned)a.b.pages) {
        const int off = slot & ((1 << a.b.page_shift) - 1);
#pragma unroll
        for (int kind = 0; kind < (Both ? 2 : 1); ++kind) {
          const bool keys = Both ? kind == 0 : item < a.Hkv;
          uint8_t* block = (uint8_t*)(keys ? a.k_pages : a.v_pages) +
                           ((size_t)page * a.b.page_units + (size_t)h * a.b.head_units) * 16 +
                           (size_t)(off - o0) * D;
          uint8_t* scale = (keys ? sc.k : sc.v) + (size_t)page * sc.stride + (size_t)h * blocks +
                           (off >> sc.block_shift);
          append_block<D, H, G>(a, live, keys, h, t, n, o0, slot, block, scale, wave % S::waves,
                                most[turn ^= 1]);
        }
      }
    }
    t += n;
  }
}

template <int D, bool H, int G, bool Both>
hipError_t append_as(const AppendArgs& a, const HeldScales& s, hipStream_t stream) {
  using S = Share<D, G>;
  const int T = a.b.T, groups = ((Both ? a.Hkv : 2 * a.Hkv) + S::heads - 1) / S::heads;
  int qsplit = 1;
  long long qblocks = 0;
  if (a.q) {
    const int units = (a.Hq + 512 / D - 1) / (512 / D);
    qsplit = std::max(1, std::min(units, (Both ? 16384 : 8192) / T));
    qblocks = ((long long)T * qsplit + kWaves - 1) / kWaves;
  }
  const int window = (long long)T * groups <= 4096 ? 1 : G;
  const long long blocks = qblocks + (long long)((T + window - 1) / window) * groups;
  append8_kernel<D, H, G, Both>
      <<<(unsigned)blocks, kThreads, 0, stream>>>(a, s, (int)qblocks, qsplit, window);
  return hipGetLastError();
}

// Both where the workgroups of one kind are more than the card takes in about one round: the
// request and page are found once for two blocks and queries begin earlier (32 and 8 heads of
// 128: 16,000 rows in blocks of 16 115 us to 101, 6000 in blocks of 32 35 to 31; but 600 in
// blocks of 8 7.4 to 13.8 and 4000 in blocks of 64 24 to 25).
template <int D, bool H, int G>
hipError_t append(const AppendArgs& a, const HeldScales& s, hipStream_t stream) {
  using S = Share<D, G>;
  const long long rows = (long long)a.b.T * ((2 * a.Hkv + S::heads - 1) / S::heads);
  return rows > 2500LL * G ? append_as<D, H, G, true>(a, s, stream)
                           : append_as<D, H, G, false>(a, s, stream);
}

// Requests of one row each (single tokens): the row's heads of queries, keys and values 512 /
// D at a time, `split` waves a row; a head's scale is that of its one row and, where slots
// from before lie in the block, of these.  (A call of 500 such rows 25 us with a
// workgroup to every head, 16 so, which is the host's.)
template <int D, bool H>
__global__ __launch_bounds__(kThreads) void append8_single_kernel(AppendArgs a, HeldScales sc,
                                                                 int split) {
  constexpr int LPH = D / 8, HPW = 64 / LPH;  // lanes of a head, heads of a wave
  const int lane = threadIdx.x & 63, e0 = (lane % LPH) * 8;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + threadIdx.x / 64);
  const int t = wave / split, part = wave % split;
  if (t >= a.b.T) return;
  const int r = request_of_row(a.b, t);
  if (r < 0) return;
  const PagedReq rq = paged_req(a.b, r);
  const int slot = rq.prefix + (t - rq.start);
  int page = slot < a.b.C ? a.b.page_table[(size_t)r * a.b.max_pages + (slot >> a.b.page_shift)] : -1;
  if ((unsigned)page >= (unsigned)a.b.pages) page = -1;
  const int off = slot & ((1 << a.b.page_shift) - 1), o0 = off & ((1 << sc.block_shift) - 1);
  const int blocks = 1 << (a.b.page_shift - sc.block_shift);  // of a page
  const bool turns = a.rope && e0 < a.rot;
  Turn turn;
  if (turns) load_turn(a, a.position ? a.position[t] : slot, e0, turn);
  const int qn = a.q ? a.Hq : 0, items = qn + 2 * a.Hkv;
  for (int i0 = part * HPW; i0 < items; i0 += split * HPW) {
    const int it = i0 + lane / LPH;
    const int kind = it < qn ? 0 : (it < qn + a.Hkv ? 1 : (it < items ? 2 : 3));
    const int h = kind == 0 ? it : (kind == 1 ? it - qn : it - qn - a.Hkv);
    const uint16_t* src = kind == 0   ? a.q + t * a.q_stride + h * D
                          : kind == 1 ? a.k + t * a.k_stride + h * D
                                      : a.v + t * a.v_stride + h * D;
    const bool held = (kind == 1 || kind == 2) && page >= 0;
    u32x4 x = {0u, 0u, 0u, 0u};
    if (kind == 0 || held) x = *(const u32x4*)(src + e0);
    uint8_t* scale = (kind == 1 ? sc.k : sc.v);
    int was = 0;
    if (held) {
      scale += (size_t)page * sc.stride + (size_t)h * blocks + (off >> sc.block_shift);
      if (o0 > 0) was = scale_in(*scale);
    }
    float y[8];
    unpack8<H>(x, y);
    norm_head<D, H>(y, kind == 0 ? a.q_norm : (kind == 1 ? a.k_norm : nullptr), a.eps, e0);
    if (a.rope) turn_head<D>(a, y, turn, e0, turns && kind < 2);
    float large = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = fabsf(y[e]);
      large = m < __builtin_inff() ? fmaxf(large, m) : large;
    }
#pragma unroll
    for (int o = 1; o < LPH; o <<= 1) large = fmaxf(large, __shfl_xor(large, o, 64));
    if (kind == 0) *(u32x4*)(a.q_out + t * a.q_out_stride + h * D + e0) = pack8<H>(y);
    if (!held) continue;
    const int now = max(scale_of(large), was);
    uint8_t* at = (uint8_t*)(kind == 1 ? a.k_pages : a.v_pages) +
                  ((size_t)page * a.b.page_units + (size_t)h * a.b.head_units) * 16 +
                  (size_t)(off - o0) * D + e0;
    const float down = scale_down(now);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= down;
    *(uint2*)(at + o0 * D) = hold8(y);
    if (now == was) continue;
    const float f = scale_up(127 - min(now - was, 126));
    for (int j = 0; j < o0; ++j) {  // the rows from before under the grown scale
      uint2* p = (uint2*)(at + j * D);
      uint2 w = *p;
      w.x = rescale4(w.x, f);
      w.y = rescale4(w.y, f);
      *p = w;
    }
    if (e0 == 0) *scale = (uint8_t)now;
  }
}

template <int D, bool H>
hipError_t append_blocks(const AppendArgs& a, const HeldScales& s, hipStream_t stream) {
  if (a.b.max_rows == 1) {
    const int units = ((a.q ? a.Hq : 0) + 2 * a.Hkv + 512 / D - 1) / (512 / D);
    const int split = std::max(1, std::min(units, 8192 / a.b.T));
    const long long waves = (long long)a.b.T * split;
    append8_single_kernel<D, H>
        <<<(unsigned)((waves + kWaves - 1) / kWaves), kThreads, 0, stream>>>(a, s, split);
    return hipGetLastError();
  }
  switch (1 << s.block_shift) {
    case 8: return append<D, H, 8>(a, s, stream);
    case 16: return append<D, H, 16>(a, s, stream);
    case 32: return append<D, H, 32>(a, s, stream);
    case 64: return append<D, H, 64>(a, s, stream);
  }
  return hipErrorInvalidValue;
}

// Compaction: a wave moves the accepted rows of one (request, group, head).  All rows of
// the path are in registers before the first store.  The scale of a block that takes
// some of them is the largest of theirs and, where slots of the prefix lie in it, of
// its own; rows under a smaller one are rounded to it.  Latency bounds it, path to pages to
// scales and rows: 72 groups of 8 heads of 128 for one request 4.6 us, for eight 6.2.
template <int D>
__global__ __launch_bounds__(kThreads) void compact8_kernel(CompactHeldArgs a) {
  constexpr int LPR = D / 16, RPS = 64 / LPR;         // lanes of a row, rows of a step
  constexpr int STEPS = (PCTREE_MAX_BLOCK + 1) / RPS;  // of the longest path
  const CompactPagedArgs& c = a.c;
  const int lane = threadIdx.x & 63, req = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const long long item = (long long)blockIdx.x * kWaves + wave;
  const int len = c.accept_len[req], pre = c.prefix_len[req];
  const long long capacity = (long long)c.max_pages << c.page_shift;
  if (item >= (long long)c.groups * c.heads || len < 0 || len >= c.W || pre < 0) return;
  const int* table = c.page_table + (size_t)req * c.max_pages;
  // the path, a node to a lane, checked
  const int node = lane <= len ? c.accept_node[(size_t)req * c.W + lane] : 0;
  const int before = __shfl_up(node, 1, 64);
  bool ok = true;
  if (lane <= len)
    ok = node >= 0 && node < c.N && (lane == 0 || node > before) && (long long)pre + node < capacity;
  if (!__all(ok)) return;
  if (!__any(lane <= len && node != lane)) return;  // nothing moves
  const int src = pre + node, dst = pre + lane;
  int ps = 0, pd = 0;
  if (lane <= len) {
    ps = table[src >> c.page_shift];
    pd = table[dst >> c.page_shift];
    ok = (unsigned)ps < (unsigned)c.pages && (unsigned)pd < (unsigned)c.pages;
  }
  if (!__all(ok)) return;
  const int g = (int)(item / c.heads), h = (int)(item % c.heads);
  const int pmask = (1 << c.page_shift) - 1, blocks = 1 << (c.page_shift - a.block_shift);
  uint8_t* pool = (uint8_t*)c.pool + g * c.group_stride + ((size_t)h << c.page_shift) * D;
  uint8_t* scales = a.scale + g * a.scale_group_stride + (size_t)h * blocks;
  const auto scale_at = [&](int page, int slot) {
    return scales + page * a.scale_page_stride + ((slot & pmask) >> a.block_shift);
  };
  const int theirs = lane <= len ? scale_in(*scale_at(ps, src)) : 0;
  // (a row's place in the pool, from the lane that holds its node)
  const long long from = ps * c.page_stride + (long long)(src & pmask) * D;
  const long long to = pd * c.page_stride + (long long)(dst & pmask) * D;
  const int sub = lane / LPR, e0 = (lane % LPR) * 16;
  u32x4 x[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
    if (s * RPS <= len)
      x[s] = *(const u32x4*)(pool + __shfl(from, min(s * RPS + sub, len), 64) + e0);
  // each destination block's scale: a maximum over the lanes of its rows
  const int b = (dst >> a.block_shift) - (pre >> a.block_shift);
  const int kept = pre & ((1 << a.block_shift) - 1);  // slots of the prefix in the first
  const int was = kept ? scale_in(*scale_at(__shfl(pd, 0, 64), pre)) : 0;
  int now = 0;
  const int last = __shfl(b, len, 64);
  for (int i = 0; i <= last; ++i) {
    int m = lane <= len && b == i ? theirs : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = max(m, __shfl_xor(m, o, 64));
    if (i == 0) m = max(m, was);
    if (b == i) now = m;
  }
  const int now0 = __shfl(now, 0, 64);
  if (kept && now0 > was) {  // the slots of the prefix under the grown scale
    const float f = scale_up(127 - min(now0 - was, 126));
    const long long base = __shfl(to, 0, 64) - (long long)kept * D;
    for (int j = sub; j < kept; j += RPS) {
      u32x4* p = (u32x4*)(pool + base + j * D + e0);
      u32x4 w = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = rescale4(w[e], f);
      *p = w;
    }
  }
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    if (s * RPS > len) break;
    const int m = s * RPS + sub, mm = min(m, len);
    const long long at = __shfl(to, mm, 64);
    const int grow = __shfl(now - theirs, mm, 64);
    const bool stays = __shfl(node, mm, 64) == mm;
    if (m > len || (stays && grow == 0)) continue;
    const float f = scale_up(127 - min(grow, 126));
    u32x4 w = x[s];
    if (grow) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = rescale4(w[e], f);
    }
    *(u32x4*)(pool + at + e0) = w;
  }
  // (the first lane of a block's rows writes its scale)
  const int b_before = __shfl_up(b, 1, 64);
  if (lane <= len && (lane == 0 || b != b_before)) *scale_at(pd, dst) = (uint8_t)now;
}

}  // namespace

hipError_t launch_append_held(const AppendArgs& a, const HeldScales& s, int D, bool f16,
                              hipStream_t stream) {
  if (D == 128)
    return f16 ? append_blocks<128, true>(a, s, stream) : append_blocks<128, false>(a, s, stream);
  return f16 ? append_blocks<64, true>(a, s, stream) : append_blocks<64, false>(a, s, stream);
}

hipError_t launch_compact_held(const CompactHeldArgs& a, hipStream_t stream) {
  const long long items = (long long)a.c.groups * a.c.heads;
  const dim3 grid((unsigned)((items + kWaves - 1) / kWaves), a.c.R);
  if (a.c.slot_units == 8) compact8_kernel<128><<<grid, kThreads, 0, stream>>>(a);
  else compact8_kernel<64><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pctree
