// Internal launcher of the sampling kernels (pctree_sample.hip), called by the C
// ABI after its argument checks.  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pctree {

// A row that pick_kernel leaves to the launches after it.
struct OpenRow {
  int state;       // 0: done; 1: by its histogram; 2: alone
  int n;           // logits of the border bin in the list
  float mx;        // the largest logit
  int bin;         // the bin in which top_p is reached
  double base;     // weights of the bins above it
  double limit;    // top_p of all weights
};

enum SampleHas { kHasTemperature = 1, kHasTopK = 2, kHasTopP = 4, kHasMinP = 8 };

struct SampleArgs {
  const void* logits;        // [T] rows, row_stride elements apart
  const float* uniform;      // [T]
  const float* temperature;  // [T] where `has` names it, else `uniform`
  const int* top_k;          // (the same for each of them)
  const float* top_p;
  const float* min_p;
  int has;
  int* token;      // [T]
  float* logprob;  // [T] or null
  float* gmax;     // [T][ng] maxima of groups of 8 << gshift elements
  double* bmass;   // [T][nb] weights of blocks of 512 elements ...
  float* bref;     // [T][nb] ... relative to this logit
  unsigned long long* hist;  // [T][bins] weights of open rows (null: no row can be open)
  unsigned long long* list;  // [T][list] keys of an open row's border bin
  OpenRow* open;             // [T]
  int* open_n;               // how many rows are left by their histograms, ...
  int* open_rows;            // [T] ... and which
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
