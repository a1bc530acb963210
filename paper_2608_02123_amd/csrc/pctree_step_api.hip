// C ABI of the norm and of what is done to logits: argument checking and the launches.
// Every check runs on the host before anything is enqueued.
#include "pctree.h"

#include "pctree_step.h"

namespace pctree {
namespace {

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr & (a - 1)) == 0; }

// A launch has at most 2^32 - 1 threads along x; a row of the norm has up to 1024.
constexpr int32_t kMaxNormRows = 1 << 21;
// A count's bits (pctree_adjust.hip); a thread's index passes a list's end by its step.
constexpr int32_t kMaxList = (1 << 29) - 1;

bool strided(int64_t stride, int64_t width, int32_t rows) {
  return stride >= width && stride % 8 == 0 && stride <= INT64_MAX / 4 / rows;
}

pctree_status check_norm(const pctree_norm* n) {
  if (!n || n->rows < 1 || n->width < 1 || n->width % 8 != 0 || !n->x || !n->out)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (n->dtype != PCTREE_BF16 && n->dtype != PCTREE_F16) return PCTREE_ERR_INVALID_ARGUMENT;
  if (n->scale && n->group != 0 && n->group != 32 && n->group != 64 && n->group != 128 &&
      n->group != 256)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!aligned(n->x, 16) || !aligned(n->weight, 16) || !aligned(n->residual, 16) ||
      !aligned(n->out, n->scale ? 8 : 16) || !aligned(n->scale, 4))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!strided(n->x_stride, n->width, n->rows) || !strided(n->out_stride, n->width, n->rows) ||
      (n->residual && !strided(n->residual_stride, n->width, n->rows)))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!(n->eps >= 0.0f) || n->eps > 3.4e38f) return PCTREE_ERR_INVALID_ARGUMENT;
  return n->width > PCTREE_MAX_NORM_WIDTH || n->rows > kMaxNormRows ? PCTREE_ERR_UNSUPPORTED
                                                                    : PCTREE_OK;
}

pctree_status check_adjust(const pctree_adjust* j) {
  if (!j || !j->logits || !j->row_start || !j->row_count || j->rows < 1 || j->vocab < 1 ||
      j->requests < 1 || j->max_rows < 1 || j->max_rows > j->rows)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (j->dtype != PCTREE_F32 && j->dtype != PCTREE_BF16 && j->dtype != PCTREE_F16)
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (j->row_stride < j->vocab || j->row_stride > INT64_MAX / 4 / j->rows)
    return PCTREE_ERR_INVALID_ARGUMENT;
  // what goes together
  const bool h = j->history, b = j->bias_token, t = j->token;
  if ((j->history_start != nullptr) != h || (j->history_count != nullptr) != h ||
      (j->prompt_count && !h) || (h ? j->history_total < 1 : j->history_total != 0) ||
      (j->bias_value != nullptr) != b || (j->bias_start != nullptr) != b ||
      (j->bias_count != nullptr) != b || (b ? j->bias_total < 1 : j->bias_total != 0) ||
      (j->mask != nullptr) != t || (t ? j->budget < 1 : j->budget != 0) ||
      (j->allowed ? j->masks < 1 : j->masks != 0 || j->allowed_row) ||
      (j->allowed && !j->allowed_row && j->masks < j->rows))
    return PCTREE_ERR_INVALID_ARGUMENT;
  if (!aligned(j->logits, j->dtype == PCTREE_F32 ? 4 : 2)) return PCTREE_ERR_INVALID_ARGUMENT;
  const void* words[] = {j->row_start,  j->row_count,  j->history,    j->history_start,
                         j->history_count, j->prompt_count, j->repetition, j->frequency,
                         j->presence,   j->bias_token, j->bias_value, j->bias_start,
                         j->bias_count, j->token,      j->mask,       j->allowed,
                         j->allowed_row};
  for (const void* p : words)
    if (!aligned(p, 4)) return PCTREE_ERR_INVALID_ARGUMENT;
  if (j->vocab > PCTREE_MAX_VOCAB || j->requests > 65535 || j->budget > PCTREE_MAX_MASK_BUDGET ||
      j->history_total > kMaxList || j->bias_total > kMaxList)
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

}  // namespace
}  // namespace pctree

using namespace pctree;

extern "C" {

pctree_status pctree_rms_norm(const pctree_norm* n, void* stream) {
  try {
    const pctree_status st = check_norm(n);
    if (st != PCTREE_OK) return st;
    NormArgs a;
    a.x = (const uint16_t*)n->x;
    a.weight = (const uint16_t*)n->weight;
    a.residual = (uint16_t*)n->residual;
    a.out = n->out;
    a.scale = n->scale;
    a.x_stride = n->x_stride;
    a.residual_stride = n->residual_stride;
    a.out_stride = n->out_stride;
    a.T = n->rows;
    a.H = n->width;
    a.group = n->scale && n->group ? n->group : n->width;
    a.groups = (n->width + a.group - 1) / a.group;
    a.eps = n->eps;
    (void)hipGetLastError();
    const hipError_t e = launch_norm(a, n->dtype == PCTREE_F16, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

pctree_status pctree_adjust_logits(const pctree_adjust* j, void* stream) {
  try {
    const pctree_status st = check_adjust(j);
    if (st != PCTREE_OK) return st;
    AdjustArgs a;
    a.logits = j->logits;
    a.row_stride = j->row_stride;
    a.T = j->rows;
    a.V = j->vocab;
    a.R = j->requests;
    a.max_rows = j->max_rows;
    a.row_start = j->row_start;
    a.row_count = j->row_count;
    a.history = j->history;
    a.history_start = j->history_start;
    a.history_count = j->history_count;
    a.prompt_count = j->prompt_count;
    a.history_total = j->history_total;
    a.repetition = j->repetition;
    a.frequency = j->frequency;
    a.presence = j->presence;
    a.bias_token = j->bias_token;
    a.bias_value = j->bias_value;
    a.bias_start = j->bias_start;
    a.bias_count = j->bias_count;
    a.bias_total = j->bias_total;
    a.token = j->token;
    a.mask = j->mask;
    a.N = j->budget;
    a.NW = (j->budget + 31) / 32;
    a.allowed = j->allowed;
    a.allowed_row = j->allowed_row;
    a.M = j->masks;
    a.AW = (j->vocab + 31) / 32;
    if (!adjust_fits(a)) return PCTREE_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    const hipError_t e = launch_adjust(a, j->dtype, (hipStream_t)stream);
    return e == hipSuccess ? PCTREE_OK : PCTREE_ERR_HIP;
  } catch (...) {
    return PCTREE_ERR_HIP;
  }
}

}  // extern "C"
