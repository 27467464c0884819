// 8-bit products of a few tokens (at most 16 rows of one matrix), with the quantisation of the rows
// in the same launch: single tokens and small decode batches, where a launch costs more
// than the bytes it moves.
//
// A block makes groups of 16 columns (16 pairs of columns for rotation and gate/up) of one 16-row MFMA
// tile.  Its waves share K by 128-byte pieces: each loads its pieces of the weights' rows
// straight into fragments (a fragment feeds one MFMA, so LDS would be a detour) and adds
// their products; the waves' sums are added in LDS (whole numbers: any order).  The rows' codes
// come from the block itself: every block quantises the tile's rows into LDS while its first
// weights are on the way.  Bound by the latency of that chain, then by the weights' bytes.
#include "gemm_kernels.hpp"
#include "i8_rows.hpp"
#include "i8_out.hpp"

namespace tr {

constexpr int FEW_ROWS = 16;
constexpr int FEW_PANEL = 48 << 10;  // bytes of codes of a tile's rows
constexpr int FEW_PAD = 16;          // between rows of codes: 16 rows at one K lie in 16 bank groups

// A row quantised by the whole block, KS waves: up to 1024 KS elements, which stay in
// registers.  red: 512 sums of squares; mred: KS entries for this row alone.
template <class P, int KS>
__device__ __forceinline__ void block_row(const P &p, const MTile &t, int r, int pitch, double *red,
                                          uint32_t *mred, int8_t *dst, float &scale) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int STEP = 512 * KS;
  const int at = threadIdx.x * 8;
  const auto row = p.row(t, r);
  float v[2][8];
#pragma unroll
  for (int q = 0; q < 2; ++q) p.load(row, at + STEP * q, v[q]);
  if constexpr (P::NORM) {
    float gv[2][8];  // (the gains on their way during the sum)
#pragma unroll
    for (int q = 0; q < 2; ++q) p.gains(at + STEP * q, gv[q]);
    // (pieces `wave` and wave + KS: of eight waves one sum, of four two)
    double s[2] = {0.0, 0.0};
    add_squares(v[0], s[0]);
    add_squares(v[1], s[KS == 8 ? 0 : 1]);
    red[threadIdx.x] = s[0];
    if constexpr (KS == 4) red[threadIdx.x + 256] = s[1];
    __syncthreads();
    const double ss = join_shared(red, lane);
    const double inv = p.inv_norm(ss);
#pragma unroll
    for (int q = 0; q < 2; ++q) norm8<typename P::elem>(gv[q], inv, v[q]);
  }
  uint32_t m = 0;
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[q][j]));
  m = wave_umax(m);
  if (lane == 0) mred[wave] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < KS; ++k) m = max(m, mred[k]);
  const RowCode rc(m);
#pragma unroll
  for (int q = 0; q < 2; ++q)
    if (at + STEP * q < pitch) *(uint2 *)(dst + at + STEP * q) = rc.code8(v[q]);
  if (threadIdx.x == 0) scale = rc.scale;
}

// The codes and scales of a tile's rows: up to two by the whole block, else a wave each.
template <class P, int KS>
__device__ __forceinline__ void tile_rows(const P &p, const MTile &t, int pitch, int8_t *panel,
                                          float *srow, double *red) {
  __shared__ uint32_t mred[2][KS];
  if (t.mvalid <= 2 && pitch <= 1024 * KS) {
    for (int r = 0; r < t.mvalid; ++r)
      block_row<P, KS>(p, t, r, pitch, red, mred[r], panel + r * (pitch + FEW_PAD), srow[r]);
  } else {
    const int lane = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < t.mvalid; r += KS) {
      const auto row = p.row(t, r);
      double inv = 0.0;
      if constexpr (P::NORM)
        inv = p.inv_norm(wave_squares([&](int c, float *v) { p.load(row, c, v); }, pitch, lane));
      const float s = wave_row(
          [&](int c, float *v) {
            p.load(row, c, v);
            if constexpr (P::NORM) {
              float gv[8];
              p.gains(c, gv);
              norm8<typename P::elem>(gv, inv, v);
            }
          },
          pitch, lane, panel + r * (pitch + FEW_PAD));
      if (lane == 0) srow[r] = s;
    }
  }
  __syncthreads();
}

// KS waves.  Block (x, y) makes tile x's column groups y, y + gridDim.y, ... of ny: the rows are
// quantised once for all of them.  A wave's first U pieces of a group are asked for ahead of the
// quantisation, or of the sums of the group before.
template <class P, int KS>
__global__ __launch_bounds__(64 * KS) void i8_few_kernel(P p, int pitch, int ny) {
  constexpr int CT = P::CT;
  constexpr int U = 4;  // pieces of a wave in flight
  extern __shared__ __align__(16) int8_t panel[];
  __shared__ i32x4_t part[KS - 1][CT][64];
  __shared__ float srow[FEW_ROWS];
  GroupScan gs;
  if constexpr (P::GROUPED) gs = group_scan(FEW_ROWS, p.cnt, p.E);
  MTile t;
  if (!p.map(blockIdx.x, FEW_ROWS, t, gs)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l15 = lane & 15, kb = 16 * (lane >> 4);
  auto group = [&](int by) {  // its first column
    if constexpr (P::CT == 2 && !P::GROUPED)
      return p.first_col(by);
    else
      return by * 16;
  };
  // piece i of this wave: bytes 128 (wave + KS i) .. of a row, two fragments
  const int np = (pitch / 128 - wave + KS - 1) / KS;
  const int8_t *w[CT];
  i32x4_t b[U][CT][2];
  auto fetch = [&](int i, i32x4_t (&f)[CT][2]) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) f[c][h] = *(const i32x4_t *)(w[c] + int64_t(i) * (128 * KS) + 64 * h);
  };
  auto start = [&](int by) {
    t.n0 = group(by);
#pragma unroll
    for (int c = 0; c < CT; ++c) w[c] = p.col_row(t, c, l15) + 128 * wave + kb;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < np) fetch(u, b[u]);
  };
  start(blockIdx.y);
  static_assert(!P::NORM || sizeof(part) >= 512 * sizeof(double), "the rows' sums lie where the products' will");
  tile_rows<P, KS>(p, t, pitch, panel, srow, (double *)part);
  // (rows past the valid ones read row 0: their sums are not stored)
  const int8_t *a = panel + (l15 < t.mvalid ? l15 : 0) * (pitch + FEW_PAD) + 128 * wave + kb;
  for (int by = blockIdx.y; by < ny; by += gridDim.y) {
    i32x4_t acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = i32x4_t{0, 0, 0, 0};
    for (int i = 0; i < np; i += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u < np) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const i32x4_t af = *(const i32x4_t *)(a + (i + u) * (128 * KS) + 64 * h);
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[c] = OpI8::mma(af, b[u][c][h], acc[c]);
          }
          if (i + u + U < np) fetch(i + u + U, b[u]);
        }
      }
    }
    const int n0 = t.n0;
    if (by + gridDim.y < ny) start(by + gridDim.y);
    if (by != blockIdx.y) __syncthreads();  // the group before has been read from part
    if (wave > 0) {
#pragma unroll
      for (int c = 0; c < CT; ++c) part[wave - 1][c][lane] = acc[c];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int k = 0; k < KS - 1; ++k)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[c] += part[k][c][lane];
      MTile o = t;
      o.n0 = n0;
      // lane: rows 4 (lane / 16) + i, column (pair) lane % 16
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * (lane >> 4) + i;
        if (r < t.mvalid) {
          if constexpr (CT == 2)
            p.store(o, r, l15, acc[0][i], acc[1][i], srow[r]);
          else
            p.store(o, r, l15, acc[0][i], srow[r]);
        }
      }
    }
  }
}

// ---------------------------------------------------------------- problems
template <typename T>
struct RowsIn {  // rows of tokens, of any stride and alignment
  typedef T elem;
  static constexpr bool NORM = false;
  const T *x;
  int64_t ldx;
  int cols;
  bool vec;
  __device__ const T *row(const MTile &, int r) const { return x + r * ldx; }
  __device__ void load(const T *row, int c, float *v) const {
    if (vec)
      row8<T, true>(row, c, cols, v);
    else
      row8<T, false>(row, c, cols, v);
  }
};

template <typename T>
struct FewLinear : RowsIn<T> {
  static constexpr int CT = 1;
  static constexpr bool GROUPED = false;
  const int8_t *w;
  const float *sw;
  T *y;
  const T *res;
  int64_t ldy, ldr;
  int N, m, pitch;
  __device__ bool map(int, int, MTile &t, const GroupScan &) const {
    t.m0 = t.e = t.p0 = 0;
    t.mvalid = N;
    return true;
  }
  __device__ const int8_t *col_row(const MTile &t, int, int c) const {
    return w + int64_t(min(t.n0 + c, m - 1)) * pitch;
  }
  __device__ void store(const MTile &t, int r, int c, int32_t v, float sr) const {
    const int col = t.n0 + c;
    if (col >= m) return;
    const float o = dequant(v, sr, sw[col]);
    put1(y + r * ldy + col, res ? Act<T>::ld(res, r * ldr + col) + o : o);
  }
};

template <typename T>
struct FewQkv : RowsIn<T> {
  static constexpr int CT = 2;
  static constexpr bool GROUPED = false;
  const int8_t *Wq, *Wk, *Wv;
  const float *sq, *sk, *sv;
  T *q, *k, *v;
  const float2 *rope;  // the rotation table, or NULL: entries are made here
  RopeJob job;
  int N, Hd, Kd, dh, pitch;
  __device__ bool map(int, int, MTile &t, const GroupScan &) const {
    t.m0 = t.e = t.p0 = 0;
    t.mvalid = N;
    return true;
  }
  // first column of 16 pairs of one head: by counts them over the heads of q, k, v
  __device__ int first_col(int by) const {
    const int per = dh / 32;
    return (by / per) * dh + (by % per) * 16;
  }
  // matrix and column within it of half `half` of pair c of the tile
  __device__ int at(const MTile &t, int half, int c, int &which) const {
    const int gc = t.n0 + c + half * (dh >> 1);
    which = gc < Hd ? 0 : gc < Hd + Kd ? 1 : 2;
    return gc - (which == 0 ? 0 : which == 1 ? Hd : Hd + Kd);
  }
  __device__ const int8_t *col_row(const MTile &t, int half, int c) const {
    int which;
    const int col = at(t, half, c, which);
    return (which == 0 ? Wq : which == 1 ? Wk : Wv) + int64_t(col) * pitch;
  }
  __device__ void store(const MTile &t, int r, int c, int32_t v1, int32_t v2, float sr) const {
    int which;
    const int col = at(t, 0, c, which), hd = dh >> 1;
    const float *s = which == 0 ? sq : which == 1 ? sk : sv;
    float y1 = dequant(v1, sr, s[col]), y2 = dequant(v2, sr, s[col + hd]);
    if (which < 2) {
      const int j = col % dh;
      const float2 cs = rope ? rope[int64_t(r) * hd + j] : rope_entry(job, r, j);
      turn(y1, y2, cs.x, cs.y);
    }
    T *o = (which == 0 ? q : which == 1 ? k : v) + int64_t(r) * (which == 0 ? Hd : Kd) + col;
    put1(o, y1);
    put1(o + hd, y2);
  }
};

// Gate/up of list rows, from the tokens: second RMSNorm (fp64, rounded once to fp32, as
// i8_norm_kernel), codes, products, h.
template <typename T>
struct FewUp {
  static constexpr int CT = 2;
  static constexpr bool GROUPED = true;
  const T *x, *g;
  const int32_t *rows, *cnt;
  int32_t *slot_of;
  const int8_t *Wg, *Wu;
  const float *sg, *su;
  float *h;
  int E, k, d, dff, pitch;
  float eps;
  __device__ bool map(int bx, int BM, MTile &t, const GroupScan &gs) const {
    return mmap_grouped(bx, BM, gs, t);
  }
  __device__ const int8_t *col_row(const MTile &t, int half, int c) const {
    return (half ? Wu : Wg) + (int64_t(t.e - 1) * dff + t.n0 + c) * pitch;
  }
  typedef T elem;
  static constexpr bool NORM = true;
  __device__ const T *row(const MTile &t, int r) const {
    const int a = rows[t.p0 + r];
    if (blockIdx.y == 0 && (threadIdx.x & 63) == 0) slot_of[a] = t.p0 + r;
    return x + int64_t(a / k) * d;
  }
  __device__ void load(const T *row, int c, float *v) const { row8<T, true>(row, c, d, v); }
  __device__ void gains(int c, float *v) const { row8<T, true>(g, c, d, v); }
  __device__ double inv_norm(double ss) const { return 1.0 / sqrt(ss / double(d) + double(eps)); }
  __device__ void store(const MTile &t, int r, int c, int32_t vg, int32_t vu, float sr) const {
    const int f = t.n0 + c;
    const int64_t wr = int64_t(t.e - 1) * dff + f;
    h[int64_t(t.p0 + r) * dff + f] = sizeof(T) == 4 ? gated64(vg, vu, sr, sg[wr], su[wr])
                                                    : gated(vg, vu, sr, sg[wr], su[wr]);
  }
};

// Down product of list rows, from h.
struct FewDown {
  typedef float elem;
  static constexpr bool NORM = false;
  static constexpr int CT = 1;
  static constexpr bool GROUPED = true;
  const float *h;
  const int32_t *cnt;
  const int8_t *Wd;
  const float *sd;
  float *Y;
  int E, d, dff, pitch;
  __device__ bool map(int bx, int BM, MTile &t, const GroupScan &gs) const {
    return mmap_grouped(bx, BM, gs, t);
  }
  __device__ const int8_t *col_row(const MTile &t, int, int c) const {
    return Wd + (int64_t(t.e - 1) * d + t.n0 + c) * pitch;
  }
  __device__ const float *row(const MTile &t, int r) const { return h + int64_t(t.p0 + r) * dff; }
  __device__ void load(const float *row, int c, float *v) const { row8<float, true>(row, c, dff, v); }
  __device__ void store(const MTile &t, int r, int c, int32_t v, float sr) const {
    const int col = t.n0 + c;
    Y[int64_t(t.p0 + r) * d + col] = dequant(v, sr, sd[int64_t(t.e - 1) * d + col]);
  }
};

// ------------------------------------------------------------------ launchers
// About two blocks a CU, one where the rows' quantisation is long (the norm; 1.3B gate/up, 1
// token: 13.8 us, two blocks 16.8, three 19.7).
template <class P>
static hipError_t launch_few(const P &p, int rows, int pitch, int tiles, int ny, hipStream_t st) {
  const size_t lds = size_t(rows) * (pitch + FEW_PAD);
  const int blocks = cu_count() * (P::NORM ? 1 : 2);
  const dim3 grid(tiles, std::max(1, std::min(ny, blocks / tiles)));
  // eight waves where K has as many pieces, or there are rows for them
  if (pitch >= 8 * 128 || rows > 4)
    i8_few_kernel<P, 8><<<grid, 512, lds, st>>>(p, pitch, ny);
  else
    i8_few_kernel<P, 4><<<grid, 256, lds, st>>>(p, pitch, ny);
  return hipGetLastError();
}

// Rows of one MFMA tile, as far as their codes fit; all of them gain by it (us, GPU, against the pass
// over the rows and the product in launches of their own): 768 -> 768, 1 token 3.6 / 7.1, 16 tokens 5.9 /
// 7.6; 2048 -> 2048, 1 token 4.0 / 10.4, 16 tokens 9.0 / 10.4; QKV 410M, 1 token 5.0 / 14.9, 16 tokens
// 9.0 / 15.1.  More rows would need several tiles a block or a grid of them, which is not built.
bool i8_few_fit(int rows, int cols) {
  return rows <= FEW_ROWS && int64_t(rows) * i8_pitch(cols) <= FEW_PANEL;
}
// Experts: up to four assignments, where every layer gains; with more experts in use the blocks of a
// wide layer are many, and each normalises its rows again (us a call of 2, 4, 6, 8, 16 assignments,
// here / in launches of their own; narrow layers would gain by more):
//   d 256,  d_ff 512    10.4 / 16.4  13.0 / 16.8  13.4 / 16.8  13.5 / 17.2
//   d 512,  d_ff 1536   11.3 / 18.7  15.9 / 19.3  18.1 / 19.5  19.1 / 19.7  20.0 / 22.5
//   d 768,  d_ff 2048   14.0 / 20.7  18.4 / 22.4  23.0 / 22.8  25.0 / 23.2  25.9 / 25.6
//   d 1024, d_ff 2816   16.8 / 23.3  22.5 / 24.5  28.4 / 24.9  32.1 / 26.0  33.3 / 29.7
//   d 2048, d_ff 5632   24.7 / 31.6  41.0 / 45.2  55.3 / 57.8  65.6 / 63.8  84.4 / 84.1
bool i8_few_fit_moe(const triroute_cfg &cfg, int N) {
  return N * cfg.top_k <= 4 && i8_few_fit(N * cfg.top_k, std::max(cfg.d_model, cfg.d_ff));
}

template <typename T>
static void rows_in(RowsIn<T> &p, const void *x, int64_t ldx, int cols) {
  p.x = (const T *)x;
  p.ldx = ldx;
  p.cols = cols;
  p.vec = cols % 8 == 0 && ((uintptr_t(x) | uintptr_t(ldx * int64_t(sizeof(T)))) & 15) == 0;
}

hipError_t i8_few_linear(int act, int N, int m, int k, const void *x, int64_t ldx, const triroute_i8_w &w,
                         const void *res, int64_t ldr, void *y, int64_t ldy, hipStream_t st) {
  auto run = [&](auto tag) {
    using T = decltype(tag);
    FewLinear<T> p;
    rows_in<T>(p, x, ldx, k);
    p.w = (const int8_t *)w.codes;
    p.sw = w.scale;
    p.y = (T *)y;
    p.res = (const T *)res;
    p.ldy = ldy;
    p.ldr = ldr;
    p.N = N;
    p.m = m;
    p.pitch = i8_pitch(k);
    return launch_few(p, N, p.pitch, 1, (m + 15) / 16, st);
  };
  return act == TRIROUTE_BF16 ? run(bf16{}) : run(float{});
}

hipError_t i8_few_qkv(const triroute_cfg &cfg, int N, const void *n1, const triroute_dense_i8_w &w,
                      const RopeJob *job, const float *rope, void *q, void *k, void *v, hipStream_t st) {
  auto run = [&](auto tag) {
    using T = decltype(tag);
    FewQkv<T> p;
    rows_in<T>(p, n1, cfg.d_model, cfg.d_model);
    p.Wq = (const int8_t *)w.Wq.codes;
    p.Wk = (const int8_t *)w.Wk.codes;
    p.Wv = (const int8_t *)w.Wv.codes;
    p.sq = w.Wq.scale;
    p.sk = w.Wk.scale;
    p.sv = w.Wv.scale;
    p.q = (T *)q;
    p.k = (T *)k;
    p.v = (T *)v;
    p.rope = (const float2 *)rope;
    if (job) p.job = *job;
    p.N = N;
    p.dh = cfg.head_dim;
    p.Hd = cfg.n_heads * cfg.head_dim;
    p.Kd = cfg.n_kv_heads * cfg.head_dim;
    p.pitch = i8_pitch(cfg.d_model);
    return launch_few(p, N, p.pitch, 1, (p.Hd + 2 * p.Kd) / 32, st);
  };
  return cfg.act == TRIROUTE_BF16 ? run(bf16{}) : run(float{});
}

hipError_t i8_few_moe(const triroute_cfg &cfg, int N, const void *xt, const void *g2,
                      const triroute_moe_i8_w &w, const triroute_compaction &c, const MoeI8Ws &ws,
                      hipStream_t st) {
  const int Nk = N * cfg.top_k, E = cfg.n_experts, d = cfg.d_model, dff = cfg.d_ff;
  auto run = [&](auto tag) {
    using T = decltype(tag);
    FewUp<T> p;
    p.x = (const T *)xt;
    p.g = (const T *)g2;
    p.rows = c.exp_rows;
    p.cnt = c.exp_cnt;
    p.slot_of = ws.slot_of;
    p.Wg = (const int8_t *)w.Wgate.codes;
    p.Wu = (const int8_t *)w.Wup.codes;
    p.sg = w.Wgate.scale;
    p.su = w.Wup.scale;
    p.h = ws.h;
    p.E = E;
    p.k = cfg.top_k;
    p.d = d;
    p.dff = dff;
    p.pitch = i8_pitch(d);
    p.eps = cfg.rms_eps;
    const hipError_t e = launch_few(p, Nk, p.pitch, std::min(E, Nk), dff / 16, st);
    if (e != hipSuccess) return e;
    FewDown q;
    q.h = ws.h;
    q.cnt = c.exp_cnt;
    q.Wd = (const int8_t *)w.Wdown.codes;
    q.sd = w.Wdown.scale;
    q.Y = ws.Y;
    q.E = E;
    q.d = d;
    q.dff = dff;
    q.pitch = i8_pitch(dff);
    return launch_few(q, Nk, q.pitch, std::min(E, Nk), d / 16, st);
  };
  return cfg.act == TRIROUTE_BF16 ? run(bf16{}) : run(float{});
}

}  // namespace tr
