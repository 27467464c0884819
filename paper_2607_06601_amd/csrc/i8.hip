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
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = max(v, uint32_t(__shfl_xor(int(v), m, WAVE)));
  return v;
}

struct RowCode {
  float a, inv, lift;
  float scale;
  bool bad;
  __device__ __forceinline__ explicit RowCode(uint32_t amax) {
    a = __uint_as_float(amax);
    bad = amax >= INF_BITS;
    scale = bad ? __uint_as_float(0x7FC00000u) : a / 127.0f;
    // 127 / a stays finite: rows of tiny values are coded 2^64 times larger (exact)
    lift = a < 1e-30f ? 18446744073709551616.0f : 1.0f;
    a *= lift;
    inv = a > 0.0f && !bad ? 127.0f / a : 0.0f;
  }
  __device__ __forceinline__ int code(float x) const {
    const float v = x * lift, t = v * inv;
    float r = rintf(t);
    // (t is off by at most 127 * 2^-22)
    if (fabsf(fabsf(t - r) - 0.5f) < 1e-4f) {
      const int k = int(fabsf(t));
      const double over = 254.0 * fabs(double(v)) - double(2 * k + 1) * double(a);
      const int c = over > 0.0 ? k + 1 : over < 0.0 ? k : k + (k & 1);
      r = copysignf(float(c), v);
    }
    return bad ? 0 : int(r);
  }
  __device__ __forceinline__ uint2 code8(const float *v) const {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[h] = (uint32_t(code(v[4 * h])) & 255u) | (uint32_t(code(v[4 * h + 1])) & 255u) << 8 |
             (uint32_t(code(v[4 * h + 2])) & 255u) << 16 | uint32_t(code(v[4 * h + 3])) << 24;
    return make_uint2(w[0], w[1]);
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
    const int64_t row = row0 + (W == 4 ? 0 : wave);
    if (W != 4 && row >= rows) break;
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
// else one wave per token, to the rows slot_of names.  Rows of up to 512 RR elements stay
// in registers; longer ones are read and normalised again for the codes.
template <typename T, bool ENTRY, int RR>
__global__ __launch_bounds__(256) void i8_norm_kernel(
    const T *__restrict__ x, const T *__restrict__ g, const int32_t *__restrict__ rows,
    const int32_t *__restrict__ off, const int32_t *__restrict__ eidx, int32_t *__restrict__ slot_of,
    int E, int k, int n, int d, int pitch, float eps, int8_t *__restrict__ codes,
    float *__restrict__ scale) {
  const int i = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int lane = threadIdx.x & 63;
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
    for (int q = 0; q < RR; ++q) row8<T, true>(xr, lane * 8 + 512 * q, d, v[q]);
#pragma unroll
    for (int q = 0; q < RR; ++q) square(v[q]);
  } else {
    for (int c = lane * 8; c < d; c += 512) {
      load8(xr + c, v[0]);
      square(v[0]);
    }
  }
  ss = wave_sum(ss);
  const double r = 1.0 / sqrt(ss / double(d) + double(eps));
  uint32_t m = 0;
  auto norm8 = [&](int c, float *w) {
    if (c >= d) return;
    float gv[8];
    load8(g + c, gv);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = float((double(w[j]) * r) * double(gv[j]));
      m = max(m, abs_bits(w[j]));
    }
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < RR; ++q) norm8(lane * 8 + 512 * q, v[q]);
  } else {
    for (int c = lane * 8; c < d; c += 512) {
      load8(xr + c, v[0]);
      norm8(c, v[0]);
    }
  }
  const RowCode rc(wave_umax(m));
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
      const int c = lane * 8 + 512 * q;
      if (c < pitch) emit(c, rc.code8(v[q]));
    }
  } else {
    for (int c = lane * 8; c < pitch; c += 512) {
      row8<T, true>(xr, c, d, v[0]);
      norm8(c, v[0]);
      emit(c, rc.code8(v[0]));
    }
  }
  if constexpr (ENTRY) {
    if (lane == 0) {
      slot_of[a] = i;
      scale[i] = rc.scale;
    }
  } else if (lane == 0) {
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
    i8_norm_kernel<T, decltype(by_entry)::value, decltype(rr)::value><<<dim3((n + 3) / 4), 256, 0, st>>>(
        (const T *)x, (const T *)g, c.exp_rows, c.exp_off, eidx, slot_of, E, k, n, d, pitch,
        cfg.rms_eps, codes, scale);
  };
  auto by_width = [&](auto tag, auto by_entry) {
    if (pitch <= 1024) run(tag, by_entry, std::integral_constant<int, 2>{});
    else if (pitch <= 2048) run(tag, by_entry, std::integral_constant<int, 4>{});
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
