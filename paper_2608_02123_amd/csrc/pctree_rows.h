// A new row's head in registers, 8 consecutive elements (e0 ..) to a lane and D / 8
// lanes to a head: norm and rotation in float32, shared by the appending kernels.
#pragma once

#include "pctree_paged.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

// cos and sin of the lane's pairs at a position (only where e0 < rot).
struct Turn {
  float cs[8], sn[8];
};
__device__ __forceinline__ void load_turn(const AppendArgs& a, int pos, int e0, Turn& t) {
  const int half = a.rot / 2;
  pos = min(max(pos, 0), a.positions - 1);
  const float* row = a.rope + (size_t)pos * a.rot;
  if (a.interleaved) {
    const f32x4 c = *(const f32x4*)(row + e0 / 2), s = *(const f32x4*)(row + half + e0 / 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t.cs[i] = c[i / 2];
      t.sn[i] = s[i / 2];
    }
  } else {
    const int p0 = e0 < half ? e0 : e0 - half;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4 c = *(const f32x4*)(row + p0 + i), s = *(const f32x4*)(row + half + p0 + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        t.cs[i + j] = c[j];
        t.sn[i + j] = s[j];
      }
    }
  }
}

template <bool H>
__device__ __forceinline__ void unpack8(u32x4 x, float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = lo16<H>(x[i]);
    y[2 * i + 1] = hi16<H>(x[i]);
  }
}
template <bool H>
__device__ __forceinline__ u32x4 pack8(const float (&y)[8]) {
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = pack16<H>(y[2 * i], y[2 * i + 1]);
  return x;
}

// y / sqrt(mean(y^2) + eps) * weight of a head (wt null: y stays; it may differ between
// the heads of a wave).
template <int D, bool H>
__device__ __forceinline__ void norm_head(float (&y)[8], const uint16_t* wt, float eps, int e0) {
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(y[i], y[i], ss);
#pragma unroll
  for (int o = 1; o < D / 8; o <<= 1) ss += __shfl_xor(ss, o, 64);
  if (wt) {
    const float inv = 1.0f / sqrtf(ss * (1.0f / D) + eps);
    const u32x4 w = *(const u32x4*)(wt + e0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = y[2 * i] * inv * lo16<H>(w[i]);
      y[2 * i + 1] = y[2 * i + 1] * inv * hi16<H>(w[i]);
    }
  }
}

// (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of a head, in the lanes where
// `turns` (every lane takes part: halves come from another lane).
template <int D>
__device__ __forceinline__ void turn_head(const AppendArgs& a, float (&y)[8], const Turn& t,
                                          int e0, bool turns) {
  const int lane = threadIdx.x & 63, half = a.rot / 2;
  float z[8];
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = i & 1 ? y[i - 1] : -y[i + 1];
  } else {
    // the lane that holds the other element of each pair
    const int partner = lane - (lane % (D / 8)) + (e0 < half ? e0 + half : e0 - half) / 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float o = __shfl(y[i], partner, 64);
      z[i] = e0 < half ? -o : o;
    }
  }
  if (turns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * t.cs[i] + z[i] * t.sn[i];
  }
}

}  // namespace
}  // namespace pctree
