// Quantisation of rows to 8-bit codes with one fp32 scale a row (the tokens of an 8-bit
// product, and weights by output channel):
//   a = max |x|,  scale = a / 127 rounded to fp32,  c = 127 x / a rounded half to even.
// The rounding is that of the exact quotient: near a border of two codes the sides are compared
// as whole numbers (254 |x| against (2 k + 1) a, both exact in fp64), so a code never
// depends on how the quotient was computed, and the same row gives the same codes on every path.
// A row that holds a NaN or an infinity gets codes 0 and scale NaN: its outputs are
// NaN, other rows' are not touched.  Codes lie in rows of i8_pitch() bytes, zero
// behind the last element, so a product needs no code of its own for the end of K.
#pragma once

#include "common.hpp"

namespace tr {

constexpr uint32_t INF_BITS = 0x7F800000u;

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Largest magnitude of a row, as the bits of |x|: as whole numbers NaN > inf > finite.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#define TR_ROR(n) uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x120 + (n), 0xF, 0xF, true))
  v = max(v, TR_ROR(1));
  v = max(v, TR_ROR(2));
  v = max(v, TR_ROR(4));
  v = max(v, TR_ROR(8));
#undef TR_ROR
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(uint32_t(a[0]), uint32_t(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(uint32_t(b[0]), uint32_t(b[1]));
}

// Scale of a row and the codes of its elements.  A code is the quotient with 1 / a in fp32, rounded; with
// one of 8 next to a border (4e-5; the quotient is off by at most 127 * 2^-23), the 8 are
// compared with their borders instead.  The quotients of a row of tiny values are of values 2^64 times
// larger (exact), so that 127 / a stays finite.
struct RowCode {
  float a, inv;
  float scale;
  bool bad, tiny;
  // amax: of the row, the same in every lane
  __device__ __forceinline__ explicit RowCode(uint32_t amax) {
    amax = __builtin_amdgcn_readfirstlane(amax);  // (so that what hangs on it branches)
    a = __uint_as_float(amax);
    bad = amax >= INF_BITS;
    tiny = amax < 0x0DA24260u;  // 1e-30
    scale = bad ? __uint_as_float(0x7FC00000u) : a / 127.0f;
    if (tiny) a *= LIFT;
    inv = a > 0.0f && !bad ? 127.0f / a : 0.0f;
  }
  static constexpr float LIFT = 18446744073709551616.0f;
  // the code of v >= 0 whose quotient is about t
  __device__ __forceinline__ int exact(float v, float t) const {
    const int k = int(t);
    if (fabsf(t - (float(k) + 0.5f)) > 1e-3f) return int(rintf(t));
    const double over = 254.0 * double(v) - double(2 * k + 1) * double(a);
    return over > 0.0 ? k + 1 : over < 0.0 ? k : k + (k & 1);
  }
  __device__ __forceinline__ uint2 code8(const float *x) const {
    float v[8], r[8], far = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
    if (tiny) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= LIFT;
    }
    // (the quotient plus 1.5 * 2^23 is rounded to a whole number, whose byte is the sum's lowest)
    constexpr float BIG = 12582912.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      r[i] = fmaf(v[i], inv, BIG);
      far = fmaxf(far, fabsf(fmaf(v[i], inv, BIG - r[i])));
    }
    if (far > 0.49996f) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        r[i] = BIG + copysignf(float(exact(fabsf(v[i]), fabsf(v[i]) * inv)), v[i]);
    }
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(r[i]);
    // bytes 0 of two words, then of two pairs
    uint2 o;
    o.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0C0C0400u),
                                __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u), 0x05040100u);
    o.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[7], w[6], 0x0C0C0400u),
                                __builtin_amdgcn_perm(w[5], w[4], 0x0C0C0400u), 0x05040100u);
    return bad ? make_uint2(0u, 0u) : o;
  }
};

// 8 elements at any element's place (the hardware takes unaligned pieces).
__device__ __forceinline__ void load8u(const bf16 *p, float *v) {
  uint32_t u[4];
  __builtin_memcpy(u, p, 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8u(const float *p, float *v) { __builtin_memcpy(v, p, 32); }

// 8 elements at c of a row of `cols`, zeros behind its end.  VEC: whole aligned pieces.
template <typename T, bool VEC>
__device__ __forceinline__ void row8(const T *row, int c, int cols, float *v) {
  if (c + 8 <= cols) {
    if constexpr (VEC) load8(row + c, v);
    else load8u(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if constexpr (!VEC) {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (c + i < cols) v[i] = Act<T>::ld(row, c + i);
    }
  }
}

// The sum of a row's squares, in fp64 and in one order whichever waves share the row, so that a
// token's normalised values are the same in every kernel: piece p of a row is its elements
// 512 p .. 512 p + 511, eight a lane; a lane adds the squares of pieces p, p + 8, p + 16, ... one
// after the other, then (join_pieces) its eight sums in pairs, and the lanes follow.
__device__ __forceinline__ void add_squares(const float *v, double &s) {
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fma(double(v[j]), double(v[j]), s);
}
// (the sums that are not there would be zeros)
template <int N>
__device__ __forceinline__ double join_pieces(const double (&s)[N]) {
  static_assert(N == 2 || N == 4 || N == 8, "whole pairs");
  if constexpr (N == 2) return s[0] + s[1];
  if constexpr (N == 4) return (s[0] + s[1]) + (s[2] + s[3]);
  if constexpr (N == 8) return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
}
// The same of sums in LDS, [8][64].
__device__ __forceinline__ double join_shared(const double *s, int lane) {
  double v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = s[64 * k + lane];
  return wave_sum(join_pieces(v));
}
// One wave's row of n elements, whose 8 values at c `load(c, v)` gives (zeros behind its end).
template <class Load>
__device__ __forceinline__ double wave_squares(const Load &load, int n, int lane) {
  double s[8] = {};
  for (int c = lane * 8; c < n; c += 4096) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (c + 512 * k >= n) continue;
      float v[8];
      load(c + 512 * k, v);
      add_squares(v, s[k]);
    }
  }
  return wave_sum(join_pieces(s));
}

// v *= g / norm for 8 elements, in fp64 and rounded once to fp32 (r: the row's 1 / norm): a product
// of a token and a gain may leave fp32 where the normalised value does not.  (bf16: that product is
// exact in fp64.  Formed in fp32, with a branch for the largest rows, the pass over 16384 tokens of 1.3B
// takes 36 us too, of 160M 19.3 instead of 20.1.)
template <typename T>
__device__ __forceinline__ void norm8(const float *gv, double r, float *v) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (sizeof(T) == 2)
      v[j] = float((double(v[j]) * double(gv[j])) * r);
    else
      v[j] = float((double(v[j]) * r) * double(gv[j]));
  }
}

// One wave quantises a row whose 8 values at c `load(c, v)` gives (zeros behind its end; it is
// called twice for each c), codes to dst[0 .. pitch); returns the row's scale.
template <class Load>
__device__ __forceinline__ float wave_row(const Load &load, int pitch, int lane, int8_t *dst) {
  uint32_t m = 0;
  for (int c = lane * 8; c < pitch; c += 512) {
    float v[8];
    load(c, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
  }
  const RowCode rc(wave_umax(m));
  for (int c = lane * 8; c < pitch; c += 512) {
    float v[8];
    load(c, v);
    *(uint2 *)(dst + c) = rc.code8(v);
  }
  return rc.scale;
}

}  // namespace tr
