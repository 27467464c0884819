// From the exact sums of an 8-bit product to its values: one form for every kernel, so that a
// token's result does not depend on the tile that made it.
#pragma once

#include "gemm_tile.hpp"

// (no product fused into a sum behind it, which the compiler would do in one kernel and not in
// another)
#pragma clang fp contract(off)

namespace tr {

__device__ __forceinline__ float dequant(int32_t v, float row, float col) {
  return float(v) * row * col;
}

// h = silu(G) U of fp32 activations: computed in fp64 and rounded once, so that the codes of h do
// not hang on the last bits of an fp32 exponential (a code one step off would move the output by far
// more than an fp32 rounding does; against bf16's rounding it does not count).
__device__ __forceinline__ float gated64(int32_t ag, int32_t au, float row, float cg, float cu) {
  const double g = double(ag) * double(row) * double(cg), u = double(au) * double(row) * double(cu);
  return float(g / (1.0 + exp(-g)) * u);
}

// h = silu(G) U of bf16 activations, in fp32: G and U are formed each with its own scales, as
// every other sum is.  (Products of the scales alone may leave fp32 where G and U do not; one of them
// for a row and one for a channel would save at most 16 of 1270 us at 1.3B, 16384 tokens.)  An exponential that
// overflows gives silu 0.
__device__ __forceinline__ float gated(int32_t ag, int32_t au, float row, float cg, float cu) {
  const float g = dequant(ag, row, cg), u = dequant(au, row, cu);
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896f * g)) * u;
}

// Rotation of the pair (a, b) by (cos, sin).
__device__ __forceinline__ void turn(float &a, float &b, float cs, float sn) {
  const float x = a, y = b;
  a = x * cs - y * sn;
  b = x * sn + y * cs;
}

// A value, rounded to the activation dtype (a NaN stays one).
__device__ __forceinline__ void put1(float *p, float v) { *p = v; }
__device__ __forceinline__ void put1(bf16 *p, float v) { *p = bf16(pk_bf16(v, v)); }

}  // namespace tr
