// Internal launcher of the sampling kernels (pctree_sample.hip), called by the C
// ABI after its argument checks.  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pctree {

struct SampleArgs {
  const void* logits;        // [T] rows, row_stride elements apart
  const float* uniform;      // [T]
  const float* temperature;  // [T] or null: 1
  const int* top_k;          // [T] or null: off
  const float* top_p;
  const float* min_p;
  int* token;      // [T]
  float* logprob;  // [T] or null
  float* gmax;     // [T][ng] maxima of groups of 64 << gshift elements
  double* bmass;   // [T][nb] weights of blocks of 512 elements ...
  float* bref;     // [T][nb] ... relative to this logit
  long long row_stride;
  int T, V;
  int ng, nb, gshift;
};

// Groups and blocks of a row of V logits at any alignment, and the workspace of T rows.
void plan_sample(int V, int* ng, int* nb, int* gshift);
size_t sample_bytes(int T, int V);
// Places gmax, bmass and bref.
void place_sample(SampleArgs* a, void* workspace);

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream);

}  // namespace pctree
