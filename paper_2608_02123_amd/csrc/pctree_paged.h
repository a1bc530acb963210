// Internal launchers of the verification step over a paged cache: new rows into
// their pages (pctree_paged.hip), attention of the new rows over the pages
// (pctree_paged_attention.hip), compaction in pages.  Called by the C ABI after
// its argument checks; not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pctree {

// The rows of a call and the pages behind them (pctree_paged_batch with the
// cache's page geometry).
struct PagedRows {
  const int* row_start;   // [R]
  const int* row_count;   // [R]
  const int* prefix_len;  // [R]
  const int* page_table;  // [R][max_pages]
  int R, max_pages, T, max_rows;
  int pages, page_shift;  // page_size = 1 << page_shift
  int C;                  // max_pages << page_shift
  uint32_t page_units;    // 16-byte units from one page to the next
  uint32_t head_units;    // 16-byte units of one head's slots in a page
};

#if defined(__HIPCC__)
// Request r's rows, clamped as the interface says (cnt 0: none).
struct PagedReq {
  int start, cnt, prefix;
};
__device__ __forceinline__ PagedReq paged_req(const PagedRows& b, int r) {
  PagedReq q;
  q.start = b.row_start[r];
  q.cnt = b.row_count[r];
  q.prefix = min(max(b.prefix_len[r], 0), b.C);
  const bool in = q.start >= 0 && q.start < b.T;
  q.cnt = in ? min(min(max(q.cnt, 0), b.max_rows), b.T - q.start) : 0;
  return q;
}

// The request of row t (the first whose rows hold it; -1: none), the same in
// every lane: the wave looks at 64 requests at a time.
__device__ __forceinline__ int request_of_row(const PagedRows& b, int t) {
  const int lane = threadIdx.x & 63;
  for (int r0 = 0; r0 < b.R; r0 += 64) {
    const int r = min(r0 + lane, b.R - 1);
    const int start = b.row_start[r], cnt = min(b.row_count[r], b.max_rows);
    const uint64_t hit = __ballot(start >= 0 && t >= start && t - start < cnt);
    if (hit) return min(r0 + (int)__builtin_ctzll(hit), b.R - 1);
  }
  return -1;
}
#endif

struct AppendArgs {
  PagedRows b;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  uint16_t* k_pages;
  uint16_t* v_pages;
  const uint16_t* q_norm;
  const uint16_t* k_norm;
  const float* rope;
  const int* position;
  long long q_stride, k_stride, v_stride, q_out_stride;
  float eps;
  int Hq, Hkv, rot, positions;
  int interleaved;
};

hipError_t launch_append(const AppendArgs& a, int D, bool f16, hipStream_t stream);

// Work split of one attention call, a pure function of sizes and the CU count.
// Requests of at most `few` rows (row count times query heads per key/value head) go
// to a kernel of their own (pctree_paged_attention.hip).
struct PagedPlan {
  int qblocks, few_qblocks;        // row blocks of a (request, kv head) at most
  int nsplit, few_nsplit;          // most slot runs of a request (1: no merge pass)
  int least;                       // slots of the shortest run (the other kernel's is fixed)
  long long blocks, few_blocks;    // workgroups (XCD-grouped, padded; 0: not launched)
  int few, few_stride;             // the most rows of such a request
  size_t parts, few_parts;         // rows of partial results
  size_t ws_bytes;
};

struct PagedAttnArgs {
  PagedRows b;
  const uint16_t* q;     // [T][Hq][D]
  const uint16_t* k;
  const uint16_t* v;
  const uint32_t* mask;  // [R][N][NW] or null: causal
  uint16_t* out;         // [T][Hq][D]
  float* part_o;         // [nsplit][T][Hq][D]
  float* part_ml;        // [nsplit][T][Hq][2]: (max of q.k, sum of weights)
  float* few_o;          // [few_nsplit][R][Hkv][few_stride][D]
  float* few_ml;         // [few_nsplit][R][Hkv][few_stride][2]
  int Hq, Hkv, g, N, NW;
  int qblocks, nsplit, least, few_qblocks, few_nsplit, few, few_stride;
  float scale_log2;
};

PagedPlan plan_paged_attention(int R, int T, int max_rows, int Hq, int Hkv, int D, int C, int cus);

// (fills in what the plan and the workspace say)
hipError_t launch_paged_attention(PagedAttnArgs a, const PagedPlan& plan, int D, bool f16,
                                  void* workspace, hipStream_t stream);

struct CompactPagedArgs {
  char* pool;
  long long group_stride, page_stride;
  int groups, pages, heads, page_shift, slot_units;
  const int* page_table;
  int max_pages;
  const int* prefix_len;
  const int* accept_node;
  const int* accept_len;
  int R, N, W;
};

hipError_t launch_compact_paged(const CompactPagedArgs& a, hipStream_t stream);

}  // namespace pctree
