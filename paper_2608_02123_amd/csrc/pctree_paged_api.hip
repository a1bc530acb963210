// C ABI of the verification step over a paged cache: argument checking and the
// launches.  Every check runs on the host before anything is enqueued.
#include "pctree.h"

#include "pctree_held.h"
#include "pctree_paged.h"
#include "pctree_sample.h"

namespace pctree {
namespace {

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr & (a - 1)) == 0; }

// Work is split for the 256 compute units of the gfx950 part, so that the
// workspace size is a function of the arguments alone.
constexpr int kPlanCUs = 256;

// A launch has at most 2^32 - 1 threads along x, in workgroups of 256.
constexpr int64_t kMaxGrid = (1 << 24) - 1;

pctree_status check_cache(const pctree_paged_cache* c) {
  if (!c || c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (c->dtype != PCTREE_BF16 && c->dtype != PCTREE_F16) return PCTREE_ERR_INVALID_ARGUMENT;
  // (a page of so many elements could pass 63 bits)
  if (c->page_stride % 8 != 0 ||
      c->page_stride / ((int64_t)c->page_size * c->head_dim) < c->kv_heads)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->page_size > PCTREE_MAX_PAGE_SIZE ||
      (c->page_size & (c->page_size - 1)) != 0 || c->kv_heads > 65535 ||
      c->page_stride / 8 > (int64_t)INT32_MAX)
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

pctree_status check_batch(const pctree_paged_cache* c, const pctree_paged_batch* b) {
  if (!b || b->requests < 1 || b->max_pages < 1 || b->rows < 1 || b->max_rows < 1 ||
      b->max_rows > b->rows)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (b->requests > 65535 || b->rows > kMaxGrid ||
      (int64_t)b->max_pages * c->page_size > PCTREE_MAX_PAGED_SLOTS)
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

pctree_status check_pointers(const pctree_paged_cache* c, const pctree_paged_batch* b) {
  if (!c->k || !c->v || !b->row_start || !b->row_count || !b->prefix_len || !b->page_table)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(b->row_start, 4) ||
      !aligned(b->row_count, 4) || !aligned(b->prefix_len, 4) || !aligned(b->page_table, 4))
    return PCTREE_ERR_INVALID_ARGUMENT;
  return PCTREE_OK;
}

// (16-byte units of a held page: half of what check_cache counts)
pctree_status check_cache8(const pctree_paged_cache8* c) {
  if (!c) return PCTREE_ERR_INVALID_ARGUMENT;
  const pctree_status st = check_cache(&c->pages);
  if (st != PCTREE_OK) return st;
  if (c->pages.page_stride % 16 != 0 || c->block < 1) return PCTREE_ERR_INVALID_ARGUMENT;
  if (c->block != 8 && c->block != 16 && c->block != 32 && c->block != 64)
    return PCTREE_ERR_UNSUPPORTED;
  if (c->block > c->pages.page_size ||
      c->scale_stride < (int64_t)c->pages.kv_heads * (c->pages.page_size / c->block) ||
      c->scale_stride > INT64_MAX / c->pages.pages)
    return PCTREE_ERR_INVALID_ARGUMENT;
  return PCTREE_OK;
}

HeldScales scales_of(const pctree_paged_cache8* c) {
  return {c->k_scale, c->v_scale, (long long)c->scale_stride,
          __builtin_ctz((unsigned)c->block)};
}

// (head dimensions are counted in 16-byte units of `unit` elements)
PagedRows rows_of(const pctree_paged_cache* c, const pctree_paged_batch* b, int unit = 8) {
  PagedRows p;
  p.row_start = b->row_start;
  p.row_count = b->row_count;
  p.prefix_len = b->prefix_len;
  p.page_table = b->page_table;
  p.R = b->requests;
  p.max_pages = b->max_pages;
  p.T = b->rows;
  p.max_rows = b->max_rows;
  p.pages = c->pages;
  p.page_shift = __builtin_ctz((unsigned)c->page_size);
  p.C = b->max_pages * c->page_size;
  p.page_units = (uint32_t)(c->page_stride / unit);
  p.head_units = (uint32_t)(c->page_size * (c->head_dim / unit));
  return p;
}

// The attention's sizes; on success the plan.
pctree_status check_attention(const pctree_paged_cache* c, const pctree_paged_batch* b,
                              int32_t q_heads, bool held, PagedPlan* plan) {
  pctree_status st = check_cache(c);
  if (st != PCTREE_OK) return st;
  st = check_batch(c, b);
  if (st != PCTREE_OK) return st;
  if (q_heads < 1 || q_heads % c->kv_heads != 0) return PCTREE_ERR_INVALID_ARGUMENT;
  // (row, head) pairs are counted in 31 bits
  if ((int64_t)b->rows * q_heads > INT32_MAX / 2) return PCTREE_ERR_UNSUPPORTED;
  *plan = plan_paged_attention(b->requests, b->rows, b->max_rows, q_heads, c->kv_heads,
                               c->head_dim, b->max_pages * c->page_size, held, kPlanCUs);
  const int hpw = 256 / c->head_dim;  // heads of a merging wave
  const int64_t row_waves = (int64_t)b->rows * ((q_heads + hpw - 1) / hpw);
  if (plan->blocks > kMaxGrid || plan->few_blocks > kMaxGrid || (row_waves + 3) / 4 > kMaxGrid)
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

// The new rows of an append; on success its arguments (but for the pages' geometry).
pctree_status check_append(const pctree_paged_cache* cache, const pctree_append* rows,
                           AppendArgs* args) {
  if (!rows || !rows->k || !rows->v || (rows->q == nullptr) != (rows->q_out == nullptr))
    return PCTREE_ERR_INVALID_ARGUMENT;
  const int64_t D = cache->head_dim, kv = cache->kv_heads * D;
  if (rows->q ? rows->q_heads < 1 : rows->q_heads != 0) return PCTREE_ERR_INVALID_ARGUMENT;
  const int64_t qn = rows->q_heads * D;
  if (rows->k_stride < kv || rows->v_stride < kv || rows->k_stride % 8 || rows->v_stride % 8 ||
      (rows->q && (rows->q_stride < qn || rows->q_out_stride < qn || rows->q_stride % 8 ||
                   rows->q_out_stride % 8)))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!aligned(rows->q, 16) || !aligned(rows->k, 16) || !aligned(rows->v, 16) ||
      !aligned(rows->q_out, 16) || !aligned(rows->q_norm, 16) || !aligned(rows->k_norm, 16) ||
      !aligned(rows->rope, 16) || !aligned(rows->position, 4))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!(rows->eps >= 0.0f) || rows->eps > 3.4e38f || rows->interleaved < 0 ||
      rows->interleaved > 1)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (rows->rope && (rows->rot_dim < 16 || rows->rot_dim % 16 != 0 || rows->rot_dim > D ||
                     rows->positions < 1))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (rows->q_heads > 65535) return PCTREE_ERR_UNSUPPORTED;
  AppendArgs& a = *args;
  a.q = (const uint16_t*)rows->q;
  a.k = (const uint16_t*)rows->k;
  a.v = (const uint16_t*)rows->v;
  a.q_out = (uint16_t*)rows->q_out;
  a.k_pages = (uint16_t*)cache->k;
  a.v_pages = (uint16_t*)cache->v;
  a.q_norm = (const uint16_t*)rows->q_norm;
  a.k_norm = (const uint16_t*)rows->k_norm;
  a.rope = rows->rope;
  a.position = rows->position;
  a.q_stride = rows->q_stride;
  a.k_stride = rows->k_stride;
  a.v_stride = rows->v_stride;
  a.q_out_stride = rows->q_out_stride;
  a.eps = rows->eps;
  a.Hq = rows->q_heads;
  a.Hkv = cache->kv_heads;
  a.rot = rows->rope ? rows->rot_dim : 0;
  a.positions = rows->positions;
  a.interleaved = rows->interleaved;
  return PCTREE_OK;
}

// The operands of an attention call; on success its arguments (but for the pages' geometry).
pctree_status check_operands(const pctree_paged_cache* cache, const PagedPlan& plan, const void* q,
                             int32_t q_heads, float scale, const uint32_t* mask, int32_t budget,
                             void* out, void* workspace, size_t workspace_bytes,
                             PagedAttnArgs* args) {
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(mask, 4) ||
      (mask && budget < 1) || !(scale > 0.0f) || scale > 3.4e38f)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (mask && budget > PCTREE_MAX_MASK_BUDGET) return PCTREE_ERR_UNSUPPORTED;
  if (plan.ws_bytes > 0 &&
      (!workspace || !aligned(workspace, 256) || workspace_bytes < plan.ws_bytes))
    return PCTREE_ERR_WORKSPACE;
  PagedAttnArgs& a = *args;
  a.s = {};
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)cache->k;
  a.v = (const uint16_t*)cache->v;
  a.mask = mask;
  a.out = (uint16_t*)out;
  a.Hq = q_heads;
  a.Hkv = cache->kv_heads;
  a.g = q_heads / cache->kv_heads;
  a.N = mask ? budget : 0;
  a.NW = (a.N + 31) / 32;
  a.scale_log2 = scale * 1.4426950408889634f;
  return PCTREE_OK;
}

// Pages in groups or groups in pages, none on another (a path's slots would be read while
// the same slots of another group are written): `block` bytes each.
bool apart(int32_t groups, int32_t pages, int64_t block, int64_t group_stride,
           int64_t page_stride) {
  return groups == 1 || (group_stride >= block && ((group_stride - block) / page_stride >= pages - 1 ||
                                                   (page_stride - block) / group_stride >= groups - 1));
}

pctree_status check_compact(void* pool, int64_t group_stride, int64_t page_stride,
                            int32_t groups, int32_t pages, int32_t heads, int32_t page_size,
                            int32_t slot_bytes, const int32_t* page_table, int32_t max_pages,
                            const int32_t* prefix_len, const int32_t* accept_node,
                            const int32_t* accept_len, int32_t requests, int32_t budget,
                            int32_t max_depth) {
  if (!pool || !page_table || !prefix_len || !accept_node || !accept_len || groups < 1 ||
      pages < 1 || heads < 1 || page_size < 1 || slot_bytes < 16 || max_pages < 1 ||
      requests < 1 || budget < 1 || max_depth < 0)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!aligned(pool, 16) || slot_bytes % 16 != 0 || group_stride % 16 != 0 ||
      page_stride % 16 != 0 || group_stride < 0 ||
      page_stride / slot_bytes < (int64_t)heads * page_size || !aligned(page_table, 4) ||
      !aligned(prefix_len, 4) || !aligned(accept_node, 4) || !aligned(accept_len, 4))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (max_depth > PCTREE_MAX_BLOCK || requests > 65535 || budget > PCTREE_MAX_MASK_BUDGET ||
      page_size > PCTREE_MAX_PAGE_SIZE || (page_size & (page_size - 1)) != 0 ||
      (int64_t)max_pages * page_size > PCTREE_MAX_PAGED_SLOTS)
    return PCTREE_ERR_UNSUPPORTED;
  // a thread for every 16 bytes of a slot in every group
  if (heads > 65535 || (int64_t)heads * (slot_bytes / 16) > INT32_MAX / groups)
    return PCTREE_ERR_UNSUPPORTED;
  return apart(groups, pages, (int64_t)heads * page_size * slot_bytes, group_stride, page_stride)
             ? PCTREE_OK
             : PCTREE_ERR_INVALID_ARGUMENT;
}

CompactPagedArgs compact_args(void* pool, int64_t group_stride, int64_t page_stride,
                              int32_t groups, int32_t pages, int32_t heads, int32_t page_size,
                              int32_t slot_bytes, const int32_t* page_table, int32_t max_pages,
                              const int32_t* prefix_len, const int32_t* accept_node,
                              const int32_t* accept_len, int32_t requests, int32_t budget,
                              int32_t max_depth) {
  CompactPagedArgs a;
  a.pool = (char*)pool;
  a.group_stride = group_stride;
  a.page_stride = page_stride;
  a.groups = groups;
  a.pages = pages;
  a.heads = heads;
  a.page_shift = __builtin_ctz((unsigned)page_size);
  a.slot_units = slot_bytes / 16;
  a.page_table = page_table;
  a.max_pages = max_pages;
  a.prefix_len = prefix_len;
  a.accept_node = accept_node;
  a.accept_len = accept_len;
  a.R = requests;
  a.N = budget;
  a.W = max_depth + 1;
  return a;
}

pctree_status check_sample(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1) return PCTREE_ERR_INVALID_ARGUMENT;
  if (vocab > PCTREE_MAX_VOCAB) return PCTREE_ERR_UNSUPPORTED;
  SampleArgs a;
  plan_sample(vocab, &a.ng, &a.nb, &a.gshift);
  return (int64_t)rows * a.nb > INT32_MAX ? PCTREE_ERR_UNSUPPORTED : PCTREE_OK;
}

}  // namespace
}  // namespace pctree

using namespace pctree;

extern "C" {

pctree_status pctree_append_paged(const pctree_paged_cache* cache, const pctree_paged_batch* batch,
                                  const pctree_append* rows, void* stream) {
  try {
    pctree_status st = check_cache(cache);
    if (st != PCTREE_OK) return st;
    st = check_batch(cache, batch);
    if (st != PCTREE_OK) return st;
    st = check_pointers(cache, batch);
    if (st != PCTREE_OK) return st;
    AppendArgs a;
    st = check_append(cache, rows, &a);
    if (st != PCTREE_OK) return st;
    a.b = rows_of(cache, batch);
    (void)hipGetLastError();
    const hipError_t e =
        launch_append(a, cache->head_dim, cache->dtype == PCTREE_F16, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

pctree_status pctree_append_paged8(const pctree_paged_cache8* cache,
                                   const pctree_paged_batch* batch, const pctree_append* rows,
                                   void* stream) {
  try {
    pctree_status st = check_cache8(cache);
    if (st != PCTREE_OK) return st;
    const pctree_paged_cache* pages = &cache->pages;
    st = check_batch(pages, batch);
    if (st != PCTREE_OK) return st;
    st = check_pointers(pages, batch);
    if (st != PCTREE_OK) return st;
    if (!cache->k_scale || !cache->v_scale) return PCTREE_ERR_INVALID_ARGUMENT;
    AppendArgs a;
    st = check_append(pages, rows, &a);
    if (st != PCTREE_OK) return st;
    // (Workgroups of keys and values: at most 4096 where each takes one row, else one for
    // Share's heads of every `block` rows, so at most rows * kv_heads / 4 + 2 * kv_heads; of
    // queries one for four rows, or 4096.)
    if ((int64_t)batch->rows * pages->kv_heads > kMaxGrid) return PCTREE_ERR_UNSUPPORTED;
    a.b = rows_of(pages, batch, 16);
    (void)hipGetLastError();
    const hipError_t e = launch_append_held(a, scales_of(cache), pages->head_dim,
                                            pages->dtype == PCTREE_F16, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

size_t pctree_paged_attention_workspace_bytes(const pctree_paged_cache* cache,
                                              const pctree_paged_batch* batch, int32_t q_heads) {
  PagedPlan plan;
  return check_attention(cache, batch, q_heads, false, &plan) == PCTREE_OK ? plan.ws_bytes : 0;
}

pctree_status pctree_paged_attention(const pctree_paged_cache* cache,
                                     const pctree_paged_batch* batch, const void* q,
                                     int32_t q_heads, float scale, const uint32_t* mask,
                                     int32_t budget, void* out, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  try {
    PagedPlan plan;
    pctree_status st = check_attention(cache, batch, q_heads, false, &plan);
    if (st != PCTREE_OK) return st;
    st = check_pointers(cache, batch);
    if (st != PCTREE_OK) return st;
    PagedAttnArgs a;
    st = check_operands(cache, plan, q, q_heads, scale, mask, budget, out, workspace,
                        workspace_bytes, &a);
    if (st != PCTREE_OK) return st;
    a.b = rows_of(cache, batch);
    (void)hipGetLastError();
    const hipError_t e =
        launch_paged_attention(a, plan, cache->head_dim, cache->dtype == PCTREE_F16, false,
                               workspace, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

size_t pctree_paged_attention8_workspace_bytes(const pctree_paged_cache8* cache,
                                               const pctree_paged_batch* batch, int32_t q_heads) {
  PagedPlan plan;
  return check_cache8(cache) == PCTREE_OK &&
                 check_attention(&cache->pages, batch, q_heads, true, &plan) == PCTREE_OK
             ? plan.ws_bytes
             : 0;
}

pctree_status pctree_paged_attention8(const pctree_paged_cache8* cache,
                                      const pctree_paged_batch* batch, const void* q,
                                      int32_t q_heads, float scale, const uint32_t* mask,
                                      int32_t budget, void* out, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  try {
    PagedPlan plan;
    pctree_status st = check_cache8(cache);
    if (st != PCTREE_OK) return st;
    const pctree_paged_cache* pages = &cache->pages;
    st = check_attention(pages, batch, q_heads, true, &plan);
    if (st != PCTREE_OK) return st;
    st = check_pointers(pages, batch);
    if (st != PCTREE_OK) return st;
    if (!cache->k_scale || !cache->v_scale) return PCTREE_ERR_INVALID_ARGUMENT;
    PagedAttnArgs a;
    st = check_operands(pages, plan, q, q_heads, scale, mask, budget, out, workspace,
                        workspace_bytes, &a);
    if (st != PCTREE_OK) return st;
    a.b = rows_of(pages, batch, 16);
    a.s = scales_of(cache);
    (void)hipGetLastError();
    const hipError_t e = launch_paged_attention(
        a, plan, pages->head_dim, pages->dtype == PCTREE_F16, true, workspace, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

size_t pctree_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  return check_sample(rows, vocab) == PCTREE_OK ? sample_bytes(rows, vocab) : 0;
}

pctree_status pctree_sample(const void* logits, int32_t dtype, int32_t rows, int32_t vocab,
                            int64_t row_stride, const float* uniform, const float* temperature,
                            const int32_t* top_k, const float* top_p, const float* min_p,
                            int32_t* token, float* logprob, void* workspace,
                            size_t workspace_bytes, void* stream) {
  try {
    const pctree_status st = check_sample(rows, vocab);
    if (st != PCTREE_OK) return st;
    if (dtype != PCTREE_F32 && dtype != PCTREE_BF16 && dtype != PCTREE_F16)
      return PCTREE_ERR_INVALID_ARGUMENT;
    if (!logits || !uniform || !token || row_stride < vocab ||
        row_stride > INT64_MAX / 4 / rows || !aligned(logits, dtype == PCTREE_F32 ? 4 : 2) ||
        !aligned(uniform, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
        !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(token, 4) || !aligned(logprob, 4))
      return PCTREE_ERR_INVALID_ARGUMENT;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < sample_bytes(rows, vocab))
      return PCTREE_ERR_WORKSPACE;
    SampleArgs a;
    a.logits = logits;
    a.uniform = uniform;
    a.has = (temperature ? kHasTemperature : 0) | (top_k ? kHasTopK : 0) |
            (top_p ? kHasTopP : 0) | (min_p ? kHasMinP : 0);
    a.temperature = temperature ? temperature : uniform;
    a.top_k = top_k ? top_k : (const int32_t*)uniform;
    a.top_p = top_p ? top_p : uniform;
    a.min_p = min_p ? min_p : uniform;
    a.token = token;
    a.logprob = logprob;
    a.row_stride = row_stride;
    a.T = rows;
    a.V = vocab;
    place_sample(&a, workspace);
    (void)hipGetLastError();
    const hipError_t e = launch_sample(a, dtype, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

pctree_status pctree_compact_paged(void* pool, int64_t group_stride, int64_t page_stride,
                                   int32_t groups, int32_t pages, int32_t heads,
                                   int32_t page_size, int32_t slot_bytes,
                                   const int32_t* page_table, int32_t max_pages,
                                   const int32_t* prefix_len, const int32_t* accept_node,
                                   const int32_t* accept_len, int32_t requests, int32_t budget,
                                   int32_t max_depth, void* stream) {
  try {
    const pctree_status st = check_compact(
        pool, group_stride, page_stride, groups, pages, heads, page_size, slot_bytes, page_table,
        max_pages, prefix_len, accept_node, accept_len, requests, budget, max_depth);
    if (st != PCTREE_OK) return st;
    const CompactPagedArgs a =
        compact_args(pool, group_stride, page_stride, groups, pages, heads, page_size, slot_bytes,
                     page_table, max_pages, prefix_len, accept_node, accept_len, requests, budget,
                     max_depth);
    (void)hipGetLastError();
    const hipError_t e = launch_compact_paged(a, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

pctree_status pctree_compact_paged8(void* pool, int64_t group_stride, int64_t page_stride,
                                    uint8_t* scale, int64_t scale_group_stride,
                                    int64_t scale_page_stride, int32_t groups, int32_t pages,
                                    int32_t heads, int32_t page_size, int32_t head_dim,
                                    int32_t block, const int32_t* page_table, int32_t max_pages,
                                    const int32_t* prefix_len, const int32_t* accept_node,
                                    const int32_t* accept_len, int32_t requests, int32_t budget,
                                    int32_t max_depth, void* stream) {
  try {
    const pctree_status st = check_compact(
        pool, group_stride, page_stride, groups, pages, heads, page_size, head_dim, page_table,
        max_pages, prefix_len, accept_node, accept_len, requests, budget, max_depth);
    if (st != PCTREE_OK) return st;
    if (!scale || block < 1 || scale_group_stride < 0 ||
        scale_page_stride < (int64_t)heads * (page_size / block))
      return PCTREE_ERR_INVALID_ARGUMENT;
    if ((head_dim != 64 && head_dim != 128) ||
        (block != 8 && block != 16 && block != 32 && block != 64))
      return PCTREE_ERR_UNSUPPORTED;
    // (a wave for every head of every group)
    if (((int64_t)groups * heads + 3) / 4 > kMaxGrid) return PCTREE_ERR_UNSUPPORTED;
    if (block > page_size || !apart(groups, pages, (int64_t)heads * (page_size / block),
                                    scale_group_stride, scale_page_stride))
      return PCTREE_ERR_INVALID_ARGUMENT;
    CompactHeldArgs a;
    a.c = compact_args(pool, group_stride, page_stride, groups, pages, heads, page_size, head_dim,
                       page_table, max_pages, prefix_len, accept_node, accept_len, requests, budget,
                       max_depth);
    a.scale = scale;
    a.scale_group_stride = scale_group_stride;
    a.scale_page_stride = scale_page_stride;
    a.block_shift = __builtin_ctz((unsigned)block);
    (void)hipGetLastError();
    const hipError_t e = launch_compact_held(a, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

}  // extern "C"
