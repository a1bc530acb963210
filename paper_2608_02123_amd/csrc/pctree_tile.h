// What the attention kernels share: MFMA operand types, softmax weights in 16
// bits, LDS layouts of a chunk's K and V, waits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pctree {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kXcds = 8;  // L2 domains the dispatcher deals workgroups over
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Two floats to packed bf16 (round to nearest even), the low half first.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2 v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                  __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The same for either 16-bit type (H: float16).
template <bool H>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if constexpr (H) {
    f16x2 v;
    v[0] = (_Float16)lo;
    v[1] = (_Float16)hi;
    return __builtin_bit_cast(uint32_t, v);
  } else {
    return pack_bf16(lo, hi);
  }
}
template <bool H>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (H)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return mfma_bf16(a, b, c);
}
// A packed pair's halves as floats.
template <bool H>
__device__ __forceinline__ float lo16(uint32_t w) {
  if constexpr (H) return (float)__builtin_bit_cast(f16x2, w)[0];
  return __uint_as_float(w << 16);
}
template <bool H>
__device__ __forceinline__ float hi16(uint32_t w) {
  if constexpr (H) return (float)__builtin_bit_cast(f16x2, w)[1];
  return __uint_as_float(w & 0xffff0000u);
}

// Permutation of the 16-byte units of a K or V row in LDS (an XOR of the unit
// index).  A K fragment read takes one unit of the 16 rows {0..3, 8..11,
// 16..19, 24..27} (+ 4, + 32); with 256-byte rows all of them start in one
// bank, so the four row bits that vary choose among the 16 units (rows of 128
// bytes alternate between two halves of the banks: three bits choose among
// 8).  A V fragment read takes 32 bytes (two units) of four consecutive keys
// per lane group: pairs of units are permuted by the key's low two bits and
// its bit 3, all that fits the 8 pairs (or two of the three, D = 64).
template <int D>
__device__ __forceinline__ int k_unit(int row) {
  return D == 128 ? (row & 3) | ((row >> 1) & 12) : ((row >> 1) & 1) | ((row >> 2) & 6);
}
template <int D>
__device__ __forceinline__ int v_unit(int row) {
  return D == 128 ? ((row & 3) << 1) | (row & 8) : (row & 2) | ((row >> 1) & 4);
}

// Every vector-memory load of the wave has landed, those into LDS among them.
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}
// A workgroup barrier for LDS traffic.
__device__ __forceinline__ void lds_barrier() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// Transposing LDS read: in each 16 lanes, lanes 4 i .. 4 i + 3 address row i (16
// consecutive 16-bit values), and lane l receives column l of rows 0 .. 3.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2 read_tr(const uint16_t* src) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)src));
}

// Low `n` bits set, n in [0, 64].
__device__ __forceinline__ uint64_t low_bits(int n) {
  return n >= 64 ? ~0ull : ((1ull << n) - 1ull);
}

// Maximum over the four lanes that hold one query row (lanes l, l ^ 16,
// l ^ 32, l ^ 48), exchanged on the VALU (v_permlane{16,32}_swap return the
// lane's own value and its partner's, in a lane-dependent order that a
// maximum does not care about).
__device__ __forceinline__ float row_max4(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                   false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                   false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace
}  // namespace pctree
