// Internal launchers of what a target's step does beside its cache: the norm before a
// projection (pctree_norm.hip), penalties, biases and masks on logits (pctree_adjust.hip).
// Called by the C ABI after its argument checks; not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pctree {

struct NormArgs {
  const uint16_t* x;
  const uint16_t* weight;  // or null
  uint16_t* residual;      // or null
  void* out;               // 16 bits, or bytes where scale is given
  float* scale;            // [T][groups] or null
  long long x_stride, residual_stride, out_stride;
  int T, H, group, groups;  // group: elements of a scale
  float eps;
};
hipError_t launch_norm(const NormArgs& a, bool f16, hipStream_t stream);

struct AdjustArgs {
  void* logits;
  long long row_stride;
  int T, V, R, max_rows;
  const int* row_start;
  const int* row_count;
  const int* history;  // or null
  const int* history_start;
  const int* history_count;
  const int* prompt_count;  // or null
  int history_total;
  const float* repetition;  // [R] or null
  const float* frequency;
  const float* presence;
  const int* bias_token;  // or null
  const float* bias_value;
  const int* bias_start;
  const int* bias_count;
  int bias_total;
  const int* token;      // [R][N] or null
  const uint32_t* mask;  // [R][N][NW]
  int N, NW;
  const uint32_t* allowed;  // [M][AW] or null
  const int* allowed_row;   // [T] or null
  int M, AW;
};
// Whether a launch can have the call's workgroups.
bool adjust_fits(const AdjustArgs& a);
hipError_t launch_adjust(const AdjustArgs& a, int dtype, hipStream_t stream);

}  // namespace pctree
