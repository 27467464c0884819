// Passes that quantise rows to 8-bit codes (i8_rows.hpp): tokens and weights, the experts'
// normalised tokens, hidden rows.
#include "i8_rows.hpp"
#include "kernels.hpp"

namespace tr {

// W waves a row (4 / W rows a block), 8 consecutive elements per lane access; the first
// RR accesses of a lane stay in registers between the maximum and the codes, later ones are
// read again.
template <typename T, bool VEC, int W, int RR>
__device__ __forceinline__ void rows_body(const T *__restrict__ x, int64_t ldx, int64_t rows,
                                          const int32_t *__restrict__ d_rows, int cols, int pitch,
                                          int8_t *__restrict__ codes, float *__restrict__ scale,
                                          int64_t blocks) {
  if (d_rows) rows = min(rows, int64_t(*d_rows));
  constexpr int STEP = 512 * W;
  __shared__ uint32_t part[4];
  const int wave = threadIdx.x >> 6;
  const int at = (W == 4 ? threadIdx.x : threadIdx.x & 63) * 8;
  for (int64_t row0 = int64_t(blockIdx.x) * (4 / W); row0 < rows; row0 += blocks * (4 / W)) {
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

template <typename T, bool VEC, int W, int RR>
__global__ __launch_bounds__(256) void i8_rows_kernel(const T *__restrict__ x, int64_t ldx,
                                                      int64_t rows,
                                                      const int32_t *__restrict__ d_rows, int cols,
                                                      int pitch, int8_t *__restrict__ codes,
                                                      float *__restrict__ scale) {
  rows_body<T, VEC, W, RR>(x, ldx, rows, d_rows, cols, pitch, codes, scale, gridDim.x);
}

// Many bf16 rows of aligned pieces, of up to 512 RR elements: a wave has its next row on the way
// while it codes one (16384 rows of 2048, bf16: 22 us, a row a wave 26).
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
template <int RR>
__device__ __forceinline__ void stream_body(const bf16 *__restrict__ x, int64_t ldx, int64_t rows,
                                            int cols, int pitch, int8_t *__restrict__ codes,
                                            float *__restrict__ scale, int blocks) {
  const int at = (threadIdx.x & 63) * 8;
  const int64_t step = int64_t(blocks) * 4;
  uint4 next[RR];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int q = 0; q < RR; ++q) {
      const int c = at + 512 * q;
      if (c < cols) next[q] = *(const uint4 *)(x + row * ldx + c);
    }
  };
#pragma unroll
  for (int q = 0; q < RR; ++q) next[q] = make_uint4(0u, 0u, 0u, 0u);  // (pieces behind the row's end stay zeros)
  int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row < rows) fetch(row);
  for (; row < rows; row += step) {
    float v[RR][8];
    uint32_t m;
    u16x2_t m2 = {0, 0};  // (bf16 pairs: |x| as whole numbers of 16 bits)
#pragma unroll
    for (int q = 0; q < RR; ++q) {
      const uint32_t u[4] = {next[q].x, next[q].y, next[q].z, next[q].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2_t, u[i] & 0x7FFF7FFFu));
        v[q][2 * i] = __uint_as_float(u[i] << 16);
        v[q][2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
      }
    }
    m = uint32_t(max(m2[0], m2[1])) << 16;
    if (row + step < rows) fetch(row + step);
    const RowCode rc(wave_umax(m));
    int8_t *cr = codes + row * pitch;
#pragma unroll
    for (int q = 0; q < RR; ++q) {
      const int c = at + 512 * q;
      if (c < pitch) *(uint2 *)(cr + c) = rc.code8(v[q]);
    }
    if (at == 0) scale[row] = rc.scale;
  }
}

template <int RR>
__global__ __launch_bounds__(256) void i8_stream_kernel(const bf16 *__restrict__ x, int64_t ldx, int64_t rows,
                                                        int cols, int pitch, int8_t *__restrict__ codes,
                                                        float *__restrict__ scale) {
  stream_body<RR>(x, ldx, rows, cols, pitch, codes, scale, gridDim.x);
}

// The same of N rows in the first blocks, and in the others the rotation table that the product
// behind it reads too (a launch less: QKV 410M, 64 tokens 14.7 -> 12.4 us).  STREAM: many bf16 rows, as
// above (QKV 1.3B, 16384 tokens, this launch 27.1 -> 24.8 us).
template <typename T, bool STREAM, int W, int RR>
__global__ __launch_bounds__(256) void i8_rows_rope_kernel(const T *__restrict__ x, int N, int cols,
                                                           int pitch, int8_t *__restrict__ codes,
                                                           float *__restrict__ scale, int blocks,
                                                           RopeJob job) {
  if (int(blockIdx.x) < blocks) {
    if constexpr (STREAM) stream_body<RR>(x, cols, N, cols, pitch, codes, scale, blocks);
    else rows_body<T, true, W, RR>(x, cols, N, nullptr, cols, pitch, codes, scale, blocks);
  } else {
    const int64_t at = int64_t(blockIdx.x - blocks) * 256 + threadIdx.x;
    if (at < int64_t(N) * job.hd) job.tab[at] = rope_entry(job, int(at / job.hd), int(at % job.hd));
  }
}

// Blocks of the stream of rows, 0 where there are too few (from two rows a wave on; fp32 rows are at
// the memory's rate without).
static int stream_blocks(int64_t rows, int cols) {
  const int waves = cu_count() * 24;
  return cols <= 2048 && rows >= 2 * waves ? waves / 4 : 0;
}
template <class F>
static void by_pieces(int pitch, F run) {
  if (pitch <= 512) run(std::integral_constant<int, 1>{});
  else if (pitch <= 1024) run(std::integral_constant<int, 2>{});
  else if (pitch <= 1536) run(std::integral_constant<int, 3>{});
  else run(std::integral_constant<int, 4>{});
}

// d_rows (or NULL): a device count that ends the rows earlier
static hipError_t launch_rows(int act, int64_t rows, const int32_t *d_rows, int cols, const void *x,
                              int64_t ldx, int8_t *codes, float *scale, hipStream_t st) {
  const int es = act == TRIROUTE_BF16 ? 2 : 4, pitch = i8_pitch(cols);
  const bool vec = cols % 8 == 0 && ((uintptr_t(x) | uintptr_t(ldx * es)) & 15) == 0;
  if (const int blocks = vec && act == TRIROUTE_BF16 ? stream_blocks(rows, cols) : 0) {
    by_pieces(pitch, [&](auto rr) {
      i8_stream_kernel<decltype(rr)::value><<<dim3(blocks), 256, 0, st>>>((const bf16 *)x, ldx, rows, cols,
                                                                          pitch, codes, scale);
    });
    return hipGetLastError();
  }
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

hipError_t launch_i8_rows_rope(int act, int N, int cols, const void *x, int8_t *codes, float *scale,
                               const RopeJob &job, hipStream_t st) {
  const int pitch = i8_pitch(cols);
  const unsigned table = unsigned((int64_t(N) * job.hd + 255) / 256);
  if (const int blocks = act == TRIROUTE_BF16 ? stream_blocks(N, cols) : 0) {
    by_pieces(pitch, [&](auto rr) {
      i8_rows_rope_kernel<bf16, true, 1, decltype(rr)::value><<<dim3(blocks + table), 256, 0, st>>>(
          (const bf16 *)x, N, cols, pitch, codes, scale, blocks, job);
    });
    return hipGetLastError();
  }
  auto run = [&](auto tag, auto w) {
    using T = decltype(tag);
    constexpr int W = decltype(w)::value;
    const int blocks = int(std::min<int64_t>((int64_t(N) * W + 3) / 4, 1 << 20));
    i8_rows_rope_kernel<T, false, W, 4><<<dim3(blocks + table), 256, 0, st>>>(
        (const T *)x, N, cols, pitch, codes, scale, blocks, job);
  };
  auto by_width = [&](auto tag) {
    if (cols > 2048) run(tag, std::integral_constant<int, 4>{});
    else run(tag, std::integral_constant<int, 1>{});
  };
  if (act == TRIROUTE_BF16) by_width(bf16{});
  else by_width(float{});
  return hipGetLastError();
}

// Second RMSNorm of the experts' rows, quantised: n2 in fp64, rounded once to fp32 (the
// values that the codes are of), for the list rows of each token's real assignments.
// ENTRY: one wave per entry of the expert lists (token rows[pos] / k to row pos, and slot_of),
// else one wave per token, to the rows slot_of names.  W waves a row; rows of up to 512 W RR
// elements stay in registers, longer ones are read and normalised again for the codes.  (Few rows: four
// waves on each, 1.3B, 32 tokens, 8.4 -> 4.8 us.  Many: the arithmetic bounds it, in 64 bits, then the
// codes; the next token fetched ahead, and the gains held, gave 19.8 -> 18.8 us at 160M, 16384 tokens, and nothing
// at 1.3B, 36.6.)
template <typename T, bool ENTRY, int W, int RR>
__global__ __launch_bounds__(256) void i8_norm_kernel(
    const T *__restrict__ x, const T *__restrict__ g, const int32_t *__restrict__ rows,
    const int32_t *__restrict__ off, const int32_t *__restrict__ eidx, int32_t *__restrict__ slot_of,
    int E, int k, int n, int d, int pitch, float eps, int8_t *__restrict__ codes,
    float *__restrict__ scale) {
  constexpr int STEP = 512 * W;
  __shared__ double part[W == 4 ? 512 : 1];
  __shared__ uint32_t mpart[W];
  const int wave = threadIdx.x >> 6;
  const int i = W == 4 ? int(blockIdx.x) : __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + wave);
  const int at = (W == 4 ? threadIdx.x : threadIdx.x & 63) * 8;
  if (i >= n || (ENTRY && i >= off[E])) return;  // off[E]: end of the last list
  const int a = ENTRY ? rows[i] : 0;
  const T *xr = x + int64_t(ENTRY ? a / k : i) * d;
  constexpr bool KEEP = RR > 0;
  float v[KEEP ? RR : 1][8];
  double ss;
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < RR; ++q) row8<T, true>(xr, at + STEP * q, d, v[q]);
  }
  if constexpr (W == 4) {  // pieces `wave`, wave + 4, ...: sums `wave` and wave + 4 of the eight
    double s[2] = {0.0, 0.0};
    if constexpr (KEEP) {
#pragma unroll
      for (int q = 0; q < RR; ++q) add_squares(v[q], s[q & 1]);
    } else {
      for (int c = at; c < d; c += 2 * STEP) {
        load8(xr + c, v[0]);
        add_squares(v[0], s[0]);
        if (c + STEP >= d) break;
        load8(xr + c + STEP, v[0]);
        add_squares(v[0], s[1]);
      }
    }
    part[threadIdx.x] = s[0];
    part[threadIdx.x + 256] = s[1];
    __syncthreads();
    ss = join_shared(part, threadIdx.x & 63);
  } else if constexpr (KEEP) {
    double s[RR] = {};
#pragma unroll
    for (int q = 0; q < RR; ++q) add_squares(v[q], s[q]);
    ss = wave_sum(join_pieces(s));
  } else {
    ss = wave_squares([&](int c, float *w) { load8(xr + c, w); }, d, threadIdx.x & 63);
  }
  const double r = 1.0 / sqrt(ss / double(d) + double(eps));
  uint32_t m = 0;
  auto normed = [&](int c, float *w) {
    if (c >= d) return;
    float gv[8];
    load8(g + c, gv);
    norm8<T>(gv, r, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, abs_bits(w[j]));
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int q = 0; q < RR; ++q) normed(at + STEP * q, v[q]);
  } else {
    for (int c = at; c < d; c += STEP) {
      load8(xr + c, v[0]);
      normed(c, v[0]);
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
      normed(c, v[0]);
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
