// New rows of the target into a paged cache, and compaction after acceptance.
//
// append_kernel: for every new row, y = x / sqrt(mean(x^2) + eps) * w per head of
// q and k, then the rotation (a, b) -> (a cos - b sin, b cos + a sin) by the
// row's position; q is written beside, k and the unchanged v go to the row's
// slot.  Everything between the 16-bit load and the one 16-bit store is float32.
// It reads and writes each element once, about ten operations apiece: bytes
// bound it (8000 rows of 32 and 8 heads of 128, 198 MB: 49 us, 4.0 TB/s, and 35 where
// they are in the last-level cache; 4 us for one row, which is the chain from its request
// and page to the store).
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pctree_paged.h"
#include "pctree_rows.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / 64;

// D / 8 lanes hold a head, 8 elements (16 bytes) each, so a wave takes 512 / D
// heads at a time.  Its items are the heads of one row, q first, then k, then v.
template <int D, bool H>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a, int split) {
  constexpr int LPH = D / 8;    // lanes of a head
  constexpr int HPW = 64 / LPH;  // heads of a wave
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kAppendWaves + threadIdx.x / 64);
  const int t = wave / split, part = wave % split;
  if (t >= a.b.T) return;
  const int r = request_of_row(a.b, t);
  if (r < 0) return;
  const PagedReq rq = paged_req(a.b, r);
  const int slot = rq.prefix + (t - rq.start);
  int page = slot < a.b.C ? a.b.page_table[(size_t)r * a.b.max_pages + (slot >> a.b.page_shift)] : -1;
  if ((unsigned)page >= (unsigned)a.b.pages) page = -1;
  const int e0 = (lane % LPH) * 8;  // the lane's first element of its head

  const bool turns = a.rope && e0 < a.rot;
  Turn turn;
  if (turns) load_turn(a, a.position ? a.position[t] : slot, e0, turn);

  const int qn = a.q ? a.Hq : 0, items = qn + 2 * a.Hkv;
  for (int i0 = part * HPW; i0 < items; i0 += split * HPW) {
    const int it = i0 + lane / LPH;
    const int kind = it < qn ? 0 : (it < qn + a.Hkv ? 1 : (it < items ? 2 : 3));
    const int h = kind == 0 ? it : (kind == 1 ? it - qn : it - qn - a.Hkv);
    u32x4 x = {0u, 0u, 0u, 0u};
    const uint16_t* src = kind == 0   ? a.q + t * a.q_stride + h * D
                          : kind == 1 ? a.k + t * a.k_stride + h * D
                                      : a.v + t * a.v_stride + h * D;
    if (kind < 3 && (kind == 0 || page >= 0)) x = *(const u32x4*)(src + e0);
    float y[8];
    unpack8<H>(x, y);
    norm_head<D, H>(y, kind == 0 ? a.q_norm : (kind == 1 ? a.k_norm : nullptr), a.eps, e0);
    if (a.rope) turn_head<D>(a, y, turn, e0, turns && kind < 2);
    if (kind != 2) x = pack8<H>(y);  // (values keep their bits)
    if (kind == 0) {
      *(u32x4*)(a.q_out + t * a.q_out_stride + h * D + e0) = x;
    } else if (kind < 3 && page >= 0) {
      const size_t off = ((size_t)page * a.b.page_units + (size_t)h * a.b.head_units) * 8 +
                         (size_t)(slot & ((1 << a.b.page_shift) - 1)) * D + e0;
      *(u32x4*)((kind == 1 ? a.k_pages : a.v_pages) + off) = x;
    }
  }
}

// Compaction: 16-byte column c of (group, head): accepted node m's moves from
// slot prefix + n_m to prefix + m.  Because n_m >= m and the nodes increase, a
// slot is read before an earlier step could overwrite it (compact_kernel's
// reasoning), so a thread copies its column in path order, in batches whose
// loads all issue before their stores.  Latency bounds it, path to pages to slots:
// 2.2 us for one request's 1.2 MB, 4.9 for eight requests' 9.4 (2.8 and 11.1 with loads
// one after the other).
constexpr int kCompactThreads = 256;
constexpr int kCompactBatch = 8;

__global__ __launch_bounds__(kCompactThreads) void compact_paged_kernel(CompactPagedArgs a) {
  const int req = blockIdx.y;
  const int len = a.accept_len[req], pre = a.prefix_len[req];
  const long long capacity = (long long)a.max_pages << a.page_shift;
  if (len < 0 || len >= a.W || pre < 0) return;
  const int* nodes = a.accept_node + (size_t)req * a.W;
  const int* table = a.page_table + (size_t)req * a.max_pages;
  __shared__ long long from[PCTREE_MAX_BLOCK + 1], to[PCTREE_MAX_BLOCK + 1];  // of the moves
  // the path, checked (one wave's lanes hold its at most 64 nodes)
  const int lane = threadIdx.x & 63;
  const int node = lane <= len ? nodes[lane] : 0;
  const int before = __shfl_up(node, 1, 64);
  bool ok = true;
  if (lane <= len)
    ok = node >= 0 && node < a.N && (lane == 0 || node > before) && (long long)pre + node < capacity;
  if (!__all(ok)) return;
  const int off_mask = (1 << a.page_shift) - 1;
  const bool moves = lane <= len && node != lane;
  const uint64_t moving = __ballot(moves);
  const int n = __builtin_popcountll(moving);
  if (lane <= len) {  // (a node that stays has to lie on a slot too)
    const int s = pre + node, d = pre + lane;
    const int ps = table[s >> a.page_shift], pd = table[d >> a.page_shift];
    ok = (unsigned)ps < (unsigned)a.pages && (unsigned)pd < (unsigned)a.pages;
    if (moves && threadIdx.x < 64) {
      const int at = __builtin_popcountll(moving & ((1ull << lane) - 1));
      from[at] = ps * a.page_stride + (long long)(s & off_mask) * a.slot_units * 16;
      to[at] = pd * a.page_stride + (long long)(d & off_mask) * a.slot_units * 16;
    }
  }
  if (!__all(ok)) return;  // (every wave found the same)
  __syncthreads();
  const long long col = (long long)blockIdx.x * kCompactThreads + threadIdx.x;
  const int per_group = a.heads * a.slot_units;
  if (col >= (long long)a.groups * per_group) return;
  const int g = (int)(col / per_group), hc = (int)(col - (long long)g * per_group);
  const int h = hc / a.slot_units, c = hc % a.slot_units;
  char* base = a.pool + g * a.group_stride +
               (((long long)h << a.page_shift) * a.slot_units + c) * 16;
  for (int m0 = 0; m0 < n; m0 += kCompactBatch) {
    // (in registers: an array of the class uint4 is kept in scratch.  All eight are
    // loaded, past the end the last again: a load that a branch may skip has to wait for
    // the ones before it.)
    u32x4 v[kCompactBatch];
#pragma unroll
    for (int b = 0; b < kCompactBatch; ++b) v[b] = *(const u32x4*)(base + from[min(m0 + b, n - 1)]);
#pragma unroll
    for (int b = 0; b < kCompactBatch; ++b)
      if (b == 0 || m0 + b < n) *(u32x4*)(base + to[m0 + b]) = v[b];
  }
}

template <int D, bool H>
hipError_t append(const AppendArgs& a, hipStream_t stream) {
  const int units = ((a.q ? a.Hq : 0) + 2 * a.Hkv + 512 / D - 1) / (512 / D);
  // About 8192 waves, from one a row that goes over all its heads to one for every 512
  // elements (32 and 8 heads of 128; us at 1, 2, 4, 12 waves a row: one row 12.9, 8.0,
  // 5.6, 3.9; 1024 rows 15.6, 10.2, 8.5, 9.3; 3000 rows 21.2, 17.5, 18.2, 21.2; 8192
  // rows 35.7, 35.7, 37.7, 48.7).
  const int split = std::max(1, std::min(units, 8192 / a.b.T));
  const long long waves = (long long)a.b.T * split;
  const unsigned blocks = (unsigned)((waves + kAppendWaves - 1) / kAppendWaves);
  append_kernel<D, H><<<blocks, kAppendThreads, 0, stream>>>(a, split);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, int D, bool f16, hipStream_t stream) {
  if (D == 128) return f16 ? append<128, true>(a, stream) : append<128, false>(a, stream);
  return f16 ? append<64, true>(a, stream) : append<64, false>(a, stream);
}

hipError_t launch_compact_paged(const CompactPagedArgs& a, hipStream_t stream) {
  const long long cols = (long long)a.groups * a.heads * a.slot_units;
  const unsigned gx = (unsigned)((cols + kCompactThreads - 1) / kCompactThreads);
  compact_paged_kernel<<<dim3(gx, a.R), kCompactThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pctree
