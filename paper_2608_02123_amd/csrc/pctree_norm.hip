// Residual addition, root-mean-square norm, and an output in 16 bits or in 8 with scales:
// v = x + residual, residual <- v, y = v / sqrt(mean(v^2) + eps) * w, then y itself or, per
// group of a row, c = max |y| / 448 and y / c in e4m3.  float32 throughout, each output
// rounded once.  A row is read once and stays in registers.  Bytes bound it: 6000 rows of
// 5120 to 8 bits in groups of 128, 215 MB, 40 us, 5.3 TB/s; one row of 4096 3.5 us, its
// loads, two sums over the workgroup and the store in a chain.
#include "pctree.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pctree_held.h"
#include "pctree_step.h"
#include "pctree_tile.h"

namespace pctree {
namespace {

constexpr float kMostHeld = 448.0f;  // the largest e4m3 number

__device__ __forceinline__ float finite_abs(float y) {
  const float m = fabsf(y);
  return m < __builtin_inff() ? m : 0.0f;
}

// y / c to nearest, but for the rarest ties, from r = 1 / c (one step with the remainder; a
// division is ten instructions: 6000 rows of 5120 in groups of 128 take 50 us with it, 45 so).
__device__ __forceinline__ float divided(float y, float c, float r) {
  const float q = y * r;
  return __builtin_fmaf(__builtin_fmaf(-q, c, y), r, q);
}

// A value of every wave joined over the workgroup (the same in every lane of a wave).
template <typename Op>
__device__ __forceinline__ float join(float v, float* slots, Op op) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = op(v, __shfl_xor(v, o, 64));
  const int waves = blockDim.x / 64;
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x / 64] = v;
  __syncthreads();
  v = slots[0];
  for (int w = 1; w < waves; ++w) v = op(v, slots[w]);
  return v;
}

// A workgroup takes a row, a thread NU units of 8 elements (unit threadIdx + i * blockDim,
// so that the lanes of a wave hold neighbouring ones).
template <bool H, bool HELD, int NU>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a) {
  __shared__ float sSum[16], sMax[16];
  const int units = a.H / 8;
  const long long t = blockIdx.x;
  float v[NU][8];
  u32x4 w[NU];
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = min((int)(threadIdx.x + i * blockDim.x), units - 1);
    const u32x4 x = *(const u32x4*)(a.x + t * a.x_stride + u * 8);
    u32x4 r = {0u, 0u, 0u, 0u};
    if (a.residual) r = *(const u32x4*)(a.residual + t * a.residual_stride + u * 8);
    if (a.weight) w[i] = *(const u32x4*)(a.weight + u * 8);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[i][2 * e] = lo16<H>(x[e]);
      v[i][2 * e + 1] = hi16<H>(x[e]);
      if (a.residual) {
        v[i][2 * e] += lo16<H>(r[e]);
        v[i][2 * e + 1] += hi16<H>(r[e]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = threadIdx.x + i * blockDim.x;
    if (u >= units) continue;
    if (a.residual) {
      u32x4 r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = pack16<H>(v[i][2 * e], v[i][2 * e + 1]);
      *(u32x4*)(a.residual + t * a.residual_stride + u * 8) = r;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(v[i][e], v[i][e], ss);
  }
  ss = join(ss, sSum, [](float p, float q) { return p + q; });
  const float inv = 1.0f / sqrtf(ss / (float)a.H + a.eps);
  float most = 0.0f;  // of the thread's units of the row
  float mine[NU];     // of each
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const bool in = (int)(threadIdx.x + i * blockDim.x) < units;
    mine[i] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y = v[i][e] * inv;
      if (a.weight) y *= e & 1 ? hi16<H>(w[i][e / 2]) : lo16<H>(w[i][e / 2]);
      v[i][e] = y;
      mine[i] = fmaxf(mine[i], finite_abs(y));
    }
    if (!in) mine[i] = 0.0f;
    most = fmaxf(most, mine[i]);
  }
  const auto larger = [](float p, float q) { return fmaxf(p, q); };
  if constexpr (HELD) {
    if (a.groups == 1) most = join(most, sMax, larger);
  }
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = threadIdx.x + i * blockDim.x;
    if constexpr (HELD) {
      float m = most;
      if (a.groups > 1) {  // (a group is 4 to 32 neighbouring lanes)
        m = mine[i];
        for (int o = 1; o < a.group / 8; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
      }
      const float c = m / kMostHeld;
      if (u >= units) continue;
      const float d = c > 0.0f ? c : 1.0f;
      if (d > 1e-30f) {
        const float r = 1.0f / d;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = divided(v[i][e], d, r);
      } else {  // (whose reciprocal may not be there)
        // A subnormal c is m / 448 rounded to a few bits, so that m / c reaches 671: held as
        // 448.  (An infinity or NaN stays one.)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float q = v[i][e] / d;
          v[i][e] = fabsf(q) < __builtin_inff() ? fminf(fmaxf(q, -kMostHeld), kMostHeld) : q;
        }
      }
      *(uint2*)((uint8_t*)a.out + t * a.out_stride + u * 8) = hold8(v[i]);
      if (u * 8 % a.group == 0) a.scale[t * a.groups + u * 8 / a.group] = c;
    } else {
      if (u >= units) continue;
      u32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = pack16<H>(v[i][2 * e], v[i][2 * e + 1]);
      *(u32x4*)((uint16_t*)a.out + t * a.out_stride + u * 8) = y;
    }
  }
}

template <bool H, bool HELD>
hipError_t norm(const NormArgs& a, hipStream_t stream) {
  const int units = a.H / 8;
  // (two units a thread from 2568 elements: 6000 rows of 5120 in one group 55 us with one,
  // 45 so, 47 with three; in groups of 128 45, 40, 45)
  const int nu = units <= 320 ? 1 : units <= 1024 ? 2 : 4;
  const int threads = ((units + nu - 1) / nu + 63) / 64 * 64;
  switch (nu) {
    case 1: norm_kernel<H, HELD, 1><<<a.T, threads, 0, stream>>>(a); break;
    case 2: norm_kernel<H, HELD, 2><<<a.T, threads, 0, stream>>>(a); break;
    case 4: norm_kernel<H, HELD, 4><<<a.T, threads, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, bool f16, hipStream_t stream) {
  if (a.scale) return f16 ? norm<true, true>(a, stream) : norm<false, true>(a, stream);
  return f16 ? norm<true, false>(a, stream) : norm<false, false>(a, stream);
}

}  // namespace pctree
