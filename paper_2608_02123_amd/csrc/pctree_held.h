// Values held in 8 bits: an e4m3 number times the power of two of its block.  Helpers of
// the kernels that write and read them, and the launchers of a paged cache in 8 bits
// (pctree_held.hip).
//
// A block's scale is a byte s, 2^(s - 127).  Powers of two cost a floating format no
// precision, products with them are exact, and a held value stays what it is under
// another scale as long as it keeps within the format's normal numbers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pctree_paged.h"

namespace pctree {

// Scales that are written: 2^-111 and up, so that every held value (2^-9 of it at least)
// is a normal bfloat16, to 2^119, the last with which 448 is below bfloat16's largest.
constexpr int kLeastScale = 16, kMostScale = 246;

#if defined(__HIPCC__)
// A stored byte as one of those (others are never written).
__device__ __forceinline__ int scale_in(int s) { return min(max(s, kLeastScale), kMostScale); }
// The smallest scale with which `largest` (finite, >= 0) is at most 448: that is 1.75 *
// 2^8, so what is above 1.75 times a power of two (mantissa 0x600000) takes the next.
__device__ __forceinline__ int scale_of(float largest) {
  return scale_in((int)((__float_as_uint(largest) + 0x1fffffu) >> 23) - 8);
}
// 2^(s - 127) and its inverse, for 1 <= s <= 253.
__device__ __forceinline__ float scale_up(int s) { return __uint_as_float((uint32_t)s << 23); }
__device__ __forceinline__ float scale_down(int s) {
  return __uint_as_float((uint32_t)(254 - s) << 23);
}

// Eight floats as e4m3, to nearest even, the first in the low byte.  (Infinities, NaN and
// what is beyond 464 become NaN.)
__device__ __forceinline__ uint2 hold8(const float (&y)[8]) {
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
  int b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
  return make_uint2((uint32_t)a, (uint32_t)b);
}
// Four held values times `f`, held again (f a power of two of at most 1).
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const int a = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * f, lo[1] * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * f, hi[1] * f, a, true);
}
#endif

// (a.k_pages and a.v_pages are bytes here, a.b.page_units and head_units 16 of them)
hipError_t launch_append_held(const AppendArgs& a, const HeldScales& s, int D, bool f16,
                              hipStream_t stream);

// c.pool and its strides as for launch_compact_paged; scale in the same order.
struct CompactHeldArgs {
  CompactPagedArgs c;
  uint8_t* scale;
  long long scale_group_stride, scale_page_stride;
  int block_shift;
};
hipError_t launch_compact_held(const CompactHeldArgs& a, hipStream_t stream);

}  // namespace pctree
