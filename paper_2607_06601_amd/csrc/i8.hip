// Quantisation of rows to 8-bit codes with one fp32 scale a row (the tokens of an 8-bit
// product, and weights by output channel):
//   a = max |x|,  scale = a / 127 rounded to fp32,  c = 127 x / a rounded half to even.
// The rounding is that of the exact quotient: near a border of two codes the sides are compared
// as whole numbers (254 |x| against (2 k + 1) a, both exact in fp64), so a code never
// depends on how the quotient was computed, and the same row gives the same codes on every path.
// A row that holds a NaN or an infinity gets codes 0 and scale NaN: its outputs are
// NaN, other rows' are not touched.  Codes lie in rows of i8_pitch() bytes, zero
// behind the last element, so a product needs no code of its own for the end of K.
#include "kernels.hpp"

namespace tr {

constexpr uint32_t INF_BITS = 0x7F800000u;

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Largest magnitude of a row, as the bits of |x|: as whole numbers NaN > inf > finite.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#define TR_ROR(n) uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x120 + (n), 0xF, 0xF, false))
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

// Scale of a row and the codes of its elements.  A code is the quotient in fp32, rounded; with
// one of 8 next to a border (4e-5; the quotient is off by at most 127 * 2^-23), the 8 are
// compared with their borders instead.  The quotients of a row of tiny values are of values 2^64 times
// larger (exact), so that 127 / a stays finite.
struct RowCode {
  float a, inv;
  float scale;
  bool bad, tiny;
  __device__ __forceinline__ explicit RowCode(uint32_t amax) {
    a = __uint_as_float(amax);
    bad = amax >= INF_BITS;
    tiny = a < 1e-30f;
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
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = v[i] * inv;
      r[i] = rintf(t);
      far = fmaxf(far, fabsf(t - r[i]));
    }
    if (far > 0.49996f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = copysignf(float(exact(fabsf(v[i]), fabsf(v[i]) * inv)), v[i]);
    }
    // (the byte of a whole number up to 127 is the lowest of it plus 1.5 * 2^23)
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(r[i] + 12582912.0f);
    // bytes 0 of two words, then of two pairs
    uint2 o;
    o.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0C0C0400u),
                                __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u), 0x05040100u);
    o.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[7], w[6], 0x0C0C0400u),
                                __builtin_amdgcn_perm(w[5], w[4], 0x0C0C0400u), 0x05040100u);
    return bad ? make_uint2(0u, 0u) : o;
  }
};

// 8 elements at c of a row of `cols`, zeros behind its end.  VEC: whole aligned pieces.
template <typename T, bool VEC>
__device__ __forceinline__ void row8(const T *row, int c, int cols, float *v) {
  if constexpr (VEC) {
    if (c < cols) {
      load8(row + c, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? Act<T>::ld(row, c + i) : 0.f;
  }
}

// W waves a row (4 / W rows a block), 8 consecutive elements per lane access; the first
// RR accesses of a lane stay in registers between the maximum and the codes, later ones are
// read again.
template <typename T, bool VEC, int W, int RR>
__global__ __launch_bounds__(256) void i8_rows_kernel(const T *__restrict__ x, int64_t ldx,
                                                      int64_t rows,
                                                      const int32_t *__restrict__ d_rows, int cols,
                                                      int pitch, int8_t *__restrict__ codes,
                                                      float *__restrict__ scale) {
  if (d_rows) rows = min(rows, int64_t(*d_rows));
  constexpr int STEP = 512 * W;
  __shared__ uint32_t part[4];
  const int wave = threadIdx.x >> 6;
  const int at = (W == 4 ? threadIdx.x : threadIdx.x & 63) * 8;
  for (int64_t row0 = int64_t(blockIdx.x) * (4 / W); row0 < rows; row0 += int64_t(gridDim.x) * (4 / W)) {
    int64_t row = row0 + (W == 4 ? 0 : wave);
    if (W != 4 && row >= rows) break;
    // rows of a product just made, its last ones first: they are still in the cache behind the
    // L2s, and the product that follows begins with the codes written last
    if (d_rows) row = rows - 1 - row;
    const T *xr = x + row * ldx;
    float v[RR][8];
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < RR; ++q) row8<T, VEC>(xr, at + STEP * q, cols, v[q]);
#pragma unroll
    for (int q = 0; q < RR; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[q][i]));
    for (int c = at + STEP * RR; c < cols; c += STEP) {
      float w[8];
      row8<T, VEC>(xr, c, cols, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, abs_bits(w[i]));
    }
    m = wave_umax(m);
    if constexpr (W == 4) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) part[wave] = m;
      __syncthreads();
      m = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const RowCode rc(m);
    int8_t *cr = codes + row * pitch;
#pragma unroll
    for (int q = 0; q < RR; ++q) {
      const int c = at + STEP * q;
      if (c < pitch) *(uint2 *)(cr + c) = rc.code8(v[q]);
    }
    for (int c = at + STEP * RR; c < pitch; c += STEP) {
      float w[8];
      row8<T, VEC>(xr, c, cols, w);
      *(uint2 *)(cr + c) = rc.code8(w);
    }
    if (at == 0) scale[row] = rc.scale;
  }
}

// d_rows (or NULL): a device count that ends the rows earlier
static hipError_t launch_rows(int act, int64_t rows, const int32_t *d_rows, int cols, const void *x,
                              int64_t ldx, int8_t *codes, float *scale, hipStream_t st) {
  const int es = act == TRIROUTE_BF16 ? 2 : 4, pitch = i8_pitch(cols);
  const bool vec = cols % 8 == 0 && ((uintptr_t(x) | uintptr_t(ldx * es)) & 15) == 0;
  auto run = [&](auto tag, auto v, auto w) {
    using T = decltype(tag);
    constexpr int W = decltype(w)::value;
    const int64_t blocks = std::min<int64_t>((rows * W + 3) / 4, 1 << 20);
    i8_rows_kernel<T, decltype(v)::value, W, 4><<<dim3(unsigned(blocks)), 256, 0, st>>>(
        (const T *)x, ldx, rows, d_rows, cols, pitch, codes, scale);
  };
  auto by_width = [&](auto tag, auto v) {
    if (cols > 2048) run(tag, v, std::integral_constant<int, 4>{});
    else run(tag, v, std::integral_constant<int, 1>{});
  };
  auto by_vec = [&](auto tag) {
    if (vec) by_width(tag, std::true_type{});
    else by_width(tag, std::false_type{});
  };
  if (act == TRIROUTE_BF16) by_vec(bf16{});
  else by_vec(float{});
  return hipGetLastError();
}

hipError_t launch_i8_rows(int act, int64_t rows, int cols, const void *x, int64_t ldx, int8_t *codes,
                          float *scale, hipStream_t st) {
  return launch_rows(act, rows, nullptr, cols, x, ldx, codes, scale, st);
}

// Second RMSNorm of the experts' rows, quantised: n2 in fp64, rounded once to fp32 (the
// values that the codes are of), for the list rows of each token's real assignments.
// ENTRY: one wave per entry of the expert lists (token rows[pos] / k to row pos, and slot_of),
// else one wave per token, to the rows slot_of names.  W waves a row; rows of up to 512 W RR
// elements stay in registers, longer ones are read and normalised again for the codes.  (Few rows: four
// waves on each, 1.3B, 32 tokens, 8.4 -> 4.8 us.)
template <typename T, bool ENTRY, int W, int RR>
__global__ __launch_bounds__(256) void i8_norm_kernel(
    const T *__restrict__ x, const T *__restrict__ g, const int32_t *__restrict__ rows,
    const int32_t *__restrict__ off, const int32_t *__restrict__ eidx, int32_t *__restrict__ slot_of,
    int E, int k, int n, int d, int pitch, float eps, int8_t *__restrict__ codes,
    float *__restrict__ scale) {
  constexpr int STEP = 512 * W;
  __shared__ double part[W];
  __shared__ uint32_t mpart[W];
  const int wave = threadIdx.x >> 6;
  const int i = W == 4 ? int(blockIdx.x) : __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + wave);
  const int at = (W == 4 ? threadIdx.x : threadIdx.x & 63) * 8;
  if (i >= n || (ENTRY && i >= off[E])) return;  // off[E]: end of the last list
  const int a = ENTRY ? rows[i] : 0;
  const T *xr = x + int64_t(ENTRY ? a / k : i) * d;
  constexpr bool KEEP = RR > 0;
  float v[KEEP ? RR : 1][8];
  double ss = 0.0;
  auto square = [&](const float *w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fma(double(w[j]), double(w[j]), ss);
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < RR; ++q) row8<T, true>(xr, at + STEP * q, d, v[q]);
#pragma unroll
    for (int q = 0; q < RR; ++q) square(v[q]);
  } else {
    for (int c = at; c < d; c += STEP) {
      load8(xr + c, v[0]);
      square(v[0]);
    }
  }
  ss = wave_sum(ss);
  if constexpr (W == 4) {
    if ((threadIdx.x & 63) == 0) part[wave] = ss;
    __syncthreads();
    ss = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const double r = 1.0 / sqrt(ss / double(d) + double(eps));
  uint32_t m = 0;
  auto norm8 = [&](int c, float *w) {
    if (c >= d) return;
    float gv[8];
    load8(g + c, gv);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 2)  // (the product of two bf16 numbers is an fp32 number)
        w[j] = float(double(w[j] * gv[j]) * r);
      else
        w[j] = float((double(w[j]) * r) * double(gv[j]));
      m = max(m, abs_bits(w[j]));
    }
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < RR; ++q) norm8(at + STEP * q, v[q]);
  } else {
    for (int c = at; c < d; c += STEP) {
      load8(xr + c, v[0]);
      norm8(c, v[0]);
    }
  }
  m = wave_umax(m);
  if constexpr (W == 4) {
    if ((threadIdx.x & 63) == 0) mpart[wave] = m;
    __syncthreads();
    m = max(max(mpart[0], mpart[1]), max(mpart[2], mpart[3]));
  }
  const RowCode rc(m);
  const int32_t *ei = eidx + int64_t(i) * k, *so = slot_of + int64_t(i) * k;
  auto emit = [&](int c, const uint2 &w) {
    if constexpr (ENTRY) {
      *(uint2 *)(codes + int64_t(i) * pitch + c) = w;
    } else {
      for (int s = 0; s < k; ++s)
        if (ei[s] != 0) *(uint2 *)(codes + int64_t(so[s]) * pitch + c) = w;
    }
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < RR; ++q) {
      const int c = at + STEP * q;
      if (c < pitch) emit(c, rc.code8(v[q]));
    }
  } else {
    for (int c = at; c < pitch; c += STEP) {
      row8<T, true>(xr, c, d, v[0]);
      norm8(c, v[0]);
      emit(c, rc.code8(v[0]));
    }
  }
  if constexpr (ENTRY) {
    if (at == 0) {
      slot_of[a] = i;
      scale[i] = rc.scale;
    }
  } else if (at == 0) {
    for (int s = 0; s < k; ++s)
      if (ei[s] != 0) scale[so[s]] = rc.scale;
  }
}

hipError_t launch_i8_norm(const triroute_cfg &cfg, int N, const void *x, const void *g,
                          const triroute_compaction &c, const int32_t *eidx, int8_t *codes,
                          float *scale, int32_t *slot_of, hipStream_t st) {
  const int k = cfg.top_k, Nk = N * k, E = cfg.n_experts, d = cfg.d_model, pitch = i8_pitch(d);
  const bool entry = Nk <= 2048;  // few: a launch costs more than normalising a row twice
  if (!entry) {
    const hipError_t e = launch_moe_slot_of(c, E, Nk, slot_of, st);
    if (e != hipSuccess) return e;
  }
  const int n = entry ? Nk : N;
  auto run = [&](auto tag, auto by_entry, auto rr) {
    using T = decltype(tag);
    constexpr bool ENTRY = decltype(by_entry)::value;
    constexpr int W = ENTRY ? 4 : 1;
    i8_norm_kernel<T, ENTRY, W, decltype(rr)::value><<<dim3((n * W + 3) / 4), 256, 0, st>>>(
        (const T *)x, (const T *)g, c.exp_rows, c.exp_off, eidx, slot_of, E, k, n, d, pitch,
        cfg.rms_eps, codes, scale);
  };
  auto by_width = [&](auto tag, auto by_entry) {
    const int w = decltype(by_entry)::value ? 4 : 1;
    if (pitch <= 1024 * w) run(tag, by_entry, std::integral_constant<int, 2>{});
    else if (pitch <= 2048 * w) run(tag, by_entry, std::integral_constant<int, 4>{});
    else run(tag, by_entry, std::integral_constant<int, 0>{});
  };
  auto by_mode = [&](auto tag) {
    if (entry) by_width(tag, std::true_type{});
    else by_width(tag, std::false_type{});
  };
  if (cfg.act == TRIROUTE_BF16) by_mode(bf16{});
  else by_mode(float{});
  return hipGetLastError();
}

// Hidden rows (fp32) of the expert lists to codes; the lists' end is read on the device.
hipError_t launch_i8_hidden(const triroute_cfg &cfg, int Nk, const float *h, const int32_t *off,
                            int8_t *codes, float *scale, hipStream_t st) {
  return launch_rows(TRIROUTE_F32, Nk, off + cfg.n_experts, cfg.d_ff, h, cfg.d_ff, codes, scale, st);
}

}  // namespace tr
