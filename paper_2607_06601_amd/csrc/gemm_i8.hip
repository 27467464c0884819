// Products of 8-bit codes on gfx950 MFMA (v_mfma_i32_16x16x64_i8) on the kernels of
// gemm_kernels.hpp: both operands are rows of codes, K-contiguous, of i8_pitch(K) bytes with
// zeros at the end, and the sums are exact in int32 (K <= 2^17), so a result does not depend on
// the tile, the order or the split of its sum.  A sum becomes
//   sum * (row's scale) * (column's scale)
// in fp32, in that order, in every kernel: the same token gives the same value in any batch.
//
//   linear: y = x W^T (+ residual), any sizes and row strides
//   QKV   : [n1] x [Wq;Wk;Wv]^T, rotate-half RoPE on q and k
//   MoE-1 : h = silu(G) U per expert, fp32
//   MoE-2 : Y = h Wdown_e^T
#include "gemm_kernels.hpp"
#include "i8_out.hpp"

namespace tr {

// 8 values, rounded to the activation dtype (a NaN stays one).
__device__ __forceinline__ void put8(float *p, const float *v) { store8(p, v); }
__device__ __forceinline__ void put8(bf16 *p, const float *v) { *(u32x4_t *)p = pack8_bf16(v); }

// Sums of a wave's tile to the staged fp32 tile C, as store_acc does for bf16; lane
// column and row mapping as there.
template <class P, int MI, int NI, int TM, int TN, int LDC>
__device__ __forceinline__ void stage_i8(const P &p, const MTile &t, float *C,
                                         const i32x4_t (&acc)[MI][NI], int wm, int wn, int lane) {
  float sc[NI];
#pragma unroll
  for (int ni = 0; ni < NI; ++ni) sc[ni] = p.col_scale(t, wn * TN + ni * 16 + (lane & 15));
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wm * TM + mi * 16 + 4 * (lane >> 4) + i;
      const float sr = p.row_scale(t, r < t.mvalid ? r : 0);
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        if constexpr (P::EPI == EPI_PLAIN) {
          C[r * LDC + wn * TN + ni * 16 + (lane & 15)] = dequant(acc[mi][ni][i], sr, sc[ni]);
        } else {
          if ((ni & 3) >= 2) continue;
          int Pp, half;
          col_pair(wn * TN + ni * 16 + (lane & 15), Pp, half);
          if constexpr (P::EPI == EPI_SWIGLU) {
            C[r * LDC + Pp] = p.hidden(acc[mi][ni][i], acc[mi][ni + 2][i], sr, sc[ni], sc[ni + 2]);
          } else {
            C[r * LDC + p.ccol(Pp, 0)] = dequant(acc[mi][ni][i], sr, sc[ni]);
            C[r * LDC + p.ccol(Pp, 1)] = dequant(acc[mi][ni + 2][i], sr, sc[ni + 2]);
          }
        }
      }
    }
}

__device__ __forceinline__ float elem(const float4 &v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// v += 8 elements as they lie in memory.
struct Raw8f {
  float4 a, b;
};
__device__ __forceinline__ void add8(const uint4 &x, float *v) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] += __uint_as_float(w[i] << 16);
    v[2 * i + 1] += __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void add8(const Raw8f &x, float *v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] += elem(x.a, i);
    v[4 + i] += elem(x.b, i);
  }
}

// The address `off` bytes behind a wave-uniform one (32-bit offsets: no 64-bit sums a lane).
template <class E>
__device__ __forceinline__ E *behind(E *base, uint32_t off) {
  return (E *)((uint8_t *)base + off);
}

// Four-wave kernel: the wave's scales in LDS, its TM rows', then its TN columns'; the
// four rows of a lane in row block mi, and its columns' where it holds NI of them side by side.
template <int MI>
__device__ __forceinline__ float4 w4_rows(const float *sc, int mi, int lane) {
  return *(const float4 *)(sc + mi * 16 + 4 * (lane >> 4));
}
template <int MI, int NI>
__device__ __forceinline__ void w4_cols(const float *sc, int lane, float (&c)[NI]) {
  const float4 *p = (const float4 *)(sc + MI * 16 + NI * (lane & 15));
#pragma unroll
  for (int q = 0; q < NI / 4; ++q) {
    const float4 v = p[q];
    c[4 * q] = v.x; c[4 * q + 1] = v.y; c[4 * q + 2] = v.z; c[4 * q + 3] = v.w;
  }
}

// ---------------------------------------------------------------- problems
template <typename T, bool VEC>  // VEC: whole 16-byte pieces of y and residual
struct LinearI8 {
  typedef OpI8 Op;
  static constexpr bool WIDE = VEC;  // runs on the four-wave kernel
  static constexpr int EPI = EPI_PLAIN;
  static constexpr bool GROUPED = false;
  const int8_t *a, *w;
  const float *sa, *sw;
  T *y;
  const T *res;
  int64_t ldy, ldr;
  int N, m, pitch;
  static constexpr int out_cols(int BN) { return BN; }
  __device__ int tiles(int BM, int ny, const GroupScan &) const { return (N + BM - 1) / BM * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &) const {
    t.m0 = bx * BM;
    t.n0 = by * BN;
    t.mvalid = min(BM, N - t.m0);
    t.e = t.p0 = 0;
    return t.mvalid > 0;
  }
  __device__ const int8_t *a_row(const MTile &t, int r) const { return a + int64_t(t.m0 + r) * pitch; }
  __device__ const int8_t *b_row(const MTile &t, int n) const {
    return t.n0 + n < m ? w + int64_t(t.n0 + n) * pitch : nullptr;
  }
  __device__ float row_scale(const MTile &t, int r) const { return sa[t.m0 + r]; }
  __device__ float col_scale(const MTile &t, int n) const { return t.n0 + n < m ? sw[t.n0 + n] : 0.f; }
  // Four-wave kernel: in wave column wn, MFMA block ni, lane column c holds
  // output column NI (16 wn + c) + ni of the tile, so each lane ends with NI
  // consecutive columns of each of its rows.
  static constexpr bool DIRECT_W4 = true;
  __device__ const int8_t *a_base() const { return a; }
  __device__ static int b_pick(int) { return 0; }
  template <int TN, int K>
  __device__ const int8_t *b_base_w4(int, int) const { return w; }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.m0 + r) * uint32_t(pitch); }
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int f = t.n0 + NI * (16 * wn + c) + ni;
    return f < m ? uint32_t(f) * uint32_t(pitch) : 0u;
  }
  __device__ const float *row_scale_at(const MTile &t, int r) const { return sa + t.m0 + r; }
  // scale n of wave column wn (TN of them)
  template <int TN>
  __device__ const float *col_scale_at(const MTile &t, int wn, int n) const {
    return sw + min(t.n0 + TN * wn + n, m - 1);
  }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const i32x4_t (&acc)[MI][NI], const float *scales, int wm,
                           int wn, int lane) const {
    static_assert(NI == 8, "whole 8-column pieces");
    const int f = t.n0 + NI * (16 * wn + (lane & 15));
    if (f >= m) return;
    float sc[NI];
    w4_cols<MI>(scales, lane, sc);
    // Residual rows of AHEAD row blocks in flight, as they lie in memory (64 registers; the
    // operands' fragments are dead here): a row block that waits for its own loads spends the
    // memory's latency eight times a tile.
    constexpr int AHEAD = std::min(MI, sizeof(T) == 2 ? 4 : 2);
    typedef std::conditional_t<sizeof(T) == 2, uint4, Raw8f> raw;
    raw x[AHEAD][4];
    const bool has = res != nullptr;
    T *yt = y + t.m0 * ldy;  // (wave-uniform; the host checks that 256 rows lie within 4 GB)
    const T *rt = res + t.m0 * ldr;
    auto row0 = [&](int mi) { return wm * MI * 16 + mi * 16 + 4 * (lane >> 4); };
    auto fetch = [&](int mi) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = row0(mi) + i;
        x[mi % AHEAD][i] = *(const raw *)behind(rt, (uint32_t(r < t.mvalid ? r : 0) * uint32_t(ldr) + f) * uint32_t(sizeof(T)));
      }
    };
    if (has) {
#pragma unroll
      for (int mi = 0; mi < AHEAD; ++mi) fetch(mi);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int r0 = row0(mi);
      const float4 sr = w4_rows<MI>(scales, mi, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) v[ni] = dequant(acc[mi][ni][i], elem(sr, i), sc[ni]);
        if (has) add8(x[mi % AHEAD][i], v);
        if (r0 + i < t.mvalid)
          put8(behind(yt, (uint32_t(r0 + i) * uint32_t(ldy) + f) * uint32_t(sizeof(T))), v);
      }
      if (has && mi + AHEAD < MI) fetch(mi + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  template <int MI, int NI, int TM, int TN, int LDC>
  __device__ void stage(const MTile &t, float *C, const i32x4_t (&acc)[MI][NI], int wm, int wn,
                        int lane) const {
    stage_i8<LinearI8, MI, NI, TM, TN, LDC>(*this, t, C, acc, wm, wn, lane);
  }
  // item = 8 columns of one row
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int CC = NC / 8;
    for (int it = tid; it < BM * CC; it += NT) {
      const int r = it / CC, c8 = (it % CC) * 8, c = t.n0 + c8;
      if (r >= t.mvalid || c >= m) continue;
      const int64_t row = t.m0 + r;
      const float *cr = C + r * LDC + c8;
      if constexpr (VEC) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = cr[u];
        if (res) {
          float x[8];
          load8(res + row * ldr + c, x);
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u] += x[u];
        }
        put8(y + row * ldy + c, v);
      } else {
        for (int u = 0; u < 8 && c + u < m; ++u)
          put1(y + row * ldy + c + u, res ? Act<T>::ld(res, row * ldr + c + u) + cr[u] : cr[u]);
      }
    }
  }
};

template <typename T>
struct QkvI8 {
  typedef OpI8 Op;
  static constexpr int EPI = EPI_ROPE;
  static constexpr bool GROUPED = false;
  const int8_t *a, *Wq, *Wk, *Wv;
  const float *sa, *sq, *sk, *sv;
  T *q, *k, *v;
  const float2 *rope;  // (cos, sin) of token row, pair j at row * dh / 2 + j
  int N, pitch, Hd, Kd, dh, Ncols;
  static constexpr int out_cols(int BN) { return BN; }
  __device__ int tiles(int BM, int ny, const GroupScan &) const { return (N + BM - 1) / BM * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &) const {
    t.m0 = bx * BM;
    t.n0 = by * BN;
    t.mvalid = min(BM, N - t.m0);
    t.e = t.p0 = 0;
    return t.mvalid > 0;
  }
  // logical column (within the tile) of half `half` of pair P
  __device__ int ccol(int P, int half) const {
    const int hd = dh >> 1;
    return (P / hd) * dh + (P % hd) + half * hd;
  }
  // column of [Wq; Wk; Wv] of physical tile column n
  __device__ int col(const MTile &t, int n) const {
    int P, half;
    col_pair(n, P, half);
    return t.n0 + ccol(P, half);
  }
  __device__ const int8_t *a_row(const MTile &t, int r) const { return a + int64_t(t.m0 + r) * pitch; }
  __device__ const int8_t *b_row(const MTile &t, int n) const {
    const int gc = col(t, n);
    if (gc >= Ncols) return nullptr;
    if (gc < Hd) return Wq + int64_t(gc) * pitch;
    if (gc < Hd + Kd) return Wk + int64_t(gc - Hd) * pitch;
    return Wv + int64_t(gc - Hd - Kd) * pitch;
  }
  __device__ float row_scale(const MTile &t, int r) const { return sa[t.m0 + r]; }
  __device__ float col_scale(const MTile &t, int n) const {
    const int gc = col(t, n);
    if (gc >= Ncols) return 0.f;
    return gc < Hd ? sq[gc] : gc < Hd + Kd ? sk[gc - Hd] : sv[gc - Hd - Kd];
  }
  // Four-wave kernel, 256-column tiles: wave column wn holds 128 columns, one head of
  // d_h 128 or two of 64; lane column c has pairs j .. j + 3 of one head, blocks 2 u and
  // 2 u + 1 the first and second half of pair j + u.
  static constexpr bool DIRECT_W4 = true;
  __device__ const int8_t *a_base() const { return a; }
  // a transfer's 8 B rows are columns of one head, so of one matrix; of the two heads of d_h 64
  // every other transfer has one
  __device__ static int b_pick(int j) { return j & 1; }
  template <int TN, int K>
  __device__ const int8_t *b_base_w4(int n0, int wn) const {
    static_assert(TN == 128, "a wave's B rows are one wave column's");
    const int gc = n0 + TN * wn + (dh == 64 ? 64 * K : 0);
    return gc < Hd ? Wq : gc < Hd + Kd ? Wk : Wv;
  }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.m0 + r) * uint32_t(pitch); }
  // first column of the lane's head, and its first pair
  __device__ void w4_head(const MTile &t, int wn, int c, int &hcol, int &j) const {
    hcol = t.n0 + 128 * wn + (dh == 64 ? 64 * (c >> 3) : 0);
    j = 4 * (dh == 64 ? c & 7 : c);
  }
  template <int NI>
  __device__ int w4_col(const MTile &t, int wn, int ni, int c) const {
    int hcol, j;
    w4_head(t, wn, c, hcol, j);
    return hcol + j + (ni >> 1) + (ni & 1) * (dh >> 1);
  }
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int gc = w4_col<NI>(t, wn, ni, c);
    const int first = gc < Hd ? 0 : gc < Hd + Kd ? Hd : Hd + Kd;
    return gc < Ncols ? uint32_t(gc - first) * uint32_t(pitch) : 0u;
  }
  __device__ const float *row_scale_at(const MTile &t, int r) const { return sa + t.m0 + r; }
  template <int TN>
  __device__ const float *col_scale_at(const MTile &t, int wn, int n) const {
    const int gc = min(t.n0 + TN * wn + n, Ncols - 1);
    return gc < Hd ? sq + gc : gc < Hd + Kd ? sk + (gc - Hd) : sv + (gc - Hd - Kd);
  }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const i32x4_t (&acc)[MI][NI], const float *scales, int wm,
                           int wn, int lane) const {
    static_assert(NI == 8, "four pairs a lane");
    int hcol, j;
    w4_head(t, wn, lane & 15, hcol, j);
    if (hcol >= Ncols) return;
    const int hd = dh >> 1;
    T *out = q;
    int ld = Hd, col = hcol;
    bool rot = true;
    if (hcol >= Hd + Kd) {
      out = v; ld = Kd; col = hcol - Hd - Kd; rot = false;
    } else if (hcol >= Hd) {
      out = k; ld = Kd; col = hcol - Hd;
    }
    const float *cl = scales + MI * 16 + (hcol - t.n0 - 128 * wn) + j;
    const float4 sc1 = *(const float4 *)cl, sc2 = *(const float4 *)(cl + hd);
    // rotation entries of two row blocks in flight (as the residual rows of LinearI8)
    float4 cs[2][4][2];
    auto row0 = [&](int mi) { return wm * MI * 16 + mi * 16 + 4 * (lane >> 4); };
    auto fetch = [&](int mi) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = row0(mi) + i;
        const float4 *tb = (const float4 *)(rope + int64_t(t.m0 + (r < t.mvalid ? r : 0)) * hd + j);
        cs[mi & 1][i][0] = tb[0];
        cs[mi & 1][i][1] = tb[1];
      }
    };
    if (rot) {
      fetch(0);
      fetch(1);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int r0 = row0(mi);
      const float4 sr = w4_rows<MI>(scales, mi, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y1[4], y2[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          y1[u] = dequant(acc[mi][2 * u][i], elem(sr, i), elem(sc1, u));
          y2[u] = dequant(acc[mi][2 * u + 1][i], elem(sr, i), elem(sc2, u));
          if (rot) {
            const float4 c4 = cs[mi & 1][i][u >> 1];  // (cos, sin) of pairs j + 2 (u / 2), + 1
            const float co = (u & 1) ? c4.z : c4.x, si = (u & 1) ? c4.w : c4.y;
            turn(y1[u], y2[u], co, si);
          }
        }
        if (r0 + i < t.mvalid) {
          T *o = out + int64_t(t.m0 + r0 + i) * ld + col + j;
          *(uint2 *)o = make_uint2(pk_bf16(y1[0], y1[1]), pk_bf16(y1[2], y1[3]));
          *(uint2 *)(o + hd) = make_uint2(pk_bf16(y2[0], y2[1]), pk_bf16(y2[2], y2[3]));
        }
      }
      if (rot && mi + 2 < MI) fetch(mi + 2);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  template <int MI, int NI, int TM, int TN, int LDC>
  __device__ void stage(const MTile &t, float *C, const i32x4_t (&acc)[MI][NI], int wm, int wn,
                        int lane) const {
    stage_i8<QkvI8, MI, NI, TM, TN, LDC>(*this, t, C, acc, wm, wn, lane);
  }
  // item = (row, 8 consecutive pairs of one head)
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int PC = NC / 16;  // 8-pair chunks per row
    const int hd = dh >> 1;
    for (int it = tid; it < BM * PC; it += NT) {
      const int r = it / PC, P0 = (it % PC) * 8;
      const int lc1 = (P0 / hd) * dh + (P0 % hd);
      const int c1 = t.n0 + lc1;
      if (r >= t.mvalid || c1 >= Ncols) continue;
      const int row = t.m0 + r;
      T *out;
      int ld, col;
      bool rot = true;
      if (c1 < Hd) {
        out = q; ld = Hd; col = c1;
      } else if (c1 < Hd + Kd) {
        out = k; ld = Kd; col = c1 - Hd;
      } else {
        out = v; ld = Kd; col = c1 - Hd - Kd; rot = false;
      }
      float y1[8], y2[8];
      const float *x1 = C + r * LDC + lc1, *x2 = x1 + hd;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        y1[u] = x1[u];
        y2[u] = x2[u];
      }
      if (rot) {
        const float2 *tb = rope + int64_t(row) * hd + col % hd;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          turn(y1[u], y2[u], tb[u].x, tb[u].y);
        }
      }
      T *o = out + int64_t(row) * ld + col;
      put8(o, y1);
      put8(o + hd, y2);
    }
  }
};

template <bool F64>
struct Moe1I8 {
  typedef OpI8 Op;
  static constexpr int EPI = EPI_SWIGLU;
  static constexpr bool GROUPED = true;
  const int8_t *a, *Wg, *Wu;  // a: rows in list order
  const float *sa, *sg, *su;
  float *h;
  const int32_t *cnt;
  int E, dff, pitch;
  static constexpr int out_cols(int BN) { return BN / 2; }
  __device__ int tiles(int BM, int ny, const GroupScan &gs) const { return gs.total * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &gs) const {
    t.n0 = first_unit(by, BN);
    return mmap_grouped(bx, BM, gs, t);
  }
  // BN/2 expert units per tile (gate + up columns)
  __device__ static int first_unit(int by, int BN) { return by * (BN / 2); }
  __device__ const int8_t *a_row(const MTile &t, int r) const { return a + int64_t(t.p0 + r) * pitch; }
  __device__ const int8_t *b_row(const MTile &t, int n) const {
    int P, half;
    col_pair(n, P, half);
    const int f = t.n0 + P;
    if (f >= dff) return nullptr;
    return (half ? Wu : Wg) + (int64_t(t.e - 1) * dff + f) * pitch;
  }
  __device__ float row_scale(const MTile &t, int r) const { return sa[t.p0 + r]; }
  __device__ float col_scale(const MTile &t, int n) const {
    int P, half;
    col_pair(n, P, half);
    const int f = t.n0 + P;
    return f < dff ? (half ? su : sg)[int64_t(t.e - 1) * dff + f] : 0.f;
  }
  __device__ float hidden(int32_t ag, int32_t au, float sr, float cg, float cu) const {
    if constexpr (F64)
      return gated64(ag, au, sr, cg, cu);
    else
      return gated(ag, au, sr, cg, cu);
  }
  // Four-wave kernel: in wave column wn, MFMA block ni, lane column c
  // holds expert unit (NI / 2) (16 wn + c) + ni / 2 of the tile, gate for
  // even ni and up for odd, so each lane ends with both halves of NI / 2
  // consecutive units.
  static constexpr bool DIRECT_W4 = true;
  __device__ const int8_t *a_base() const { return a; }
  // a transfer has 8 rows of one block ni: two transfers of gate rows, two of up rows, ...
  __device__ static int b_pick(int j) { return (j >> 1) & 1; }
  template <int TN, int K>
  __device__ const int8_t *b_base_w4(int, int) const { return K ? Wu : Wg; }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.p0 + r) * uint32_t(pitch); }
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int f = t.n0 + (NI / 2) * (16 * wn + c) + (ni >> 1);
    return f < dff ? uint32_t((t.e - 1) * dff + f) * uint32_t(pitch) : 0u;
  }
  __device__ const float *row_scale_at(const MTile &t, int r) const { return sa + t.p0 + r; }
  // the wave's TN / 2 gate scales, then its up scales
  template <int TN>
  __device__ const float *col_scale_at(const MTile &t, int wn, int n) const {
    const int u = n < TN / 2 ? n : n - TN / 2;
    return (n < TN / 2 ? sg : su) + (int64_t(t.e - 1) * dff + min(t.n0 + TN / 2 * wn + u, dff - 1));
  }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const i32x4_t (&acc)[MI][NI], const float *scales, int wm,
                           int wn, int lane) const {
    static_assert(NI == 8 && !F64, "4 units per lane, one 16-byte piece per row");
    const int f = t.n0 + (NI / 2) * (16 * wn + (lane & 15));
    if (f >= dff) return;  // d_ff is a multiple of 4: a lane's units are all in or all out
    const float *cl = scales + MI * 16 + (NI / 2) * (lane & 15);
    const float4 cg = *(const float4 *)cl, cu = *(const float4 *)(cl + NI * 8);
    float *out = h + int64_t(t.p0) * dff;  // (wave-uniform; a lane's offset fits 32 bits)
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int r0 = wm * MI * 16 + mi * 16 + 4 * (lane >> 4);
      const float4 sr = w4_rows<MI>(scales, mi, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          v[u] = hidden(acc[mi][2 * u][i], acc[mi][2 * u + 1][i], elem(sr, i), elem(cg, u), elem(cu, u));
        if (r0 + i < t.mvalid)
          *(float4 *)behind(out, uint32_t((r0 + i) * dff + f) * 4u) = make_float4(v[0], v[1], v[2], v[3]);
      }
    }
  }
  template <int MI, int NI, int TM, int TN, int LDC>
  __device__ void stage(const MTile &t, float *C, const i32x4_t (&acc)[MI][NI], int wm, int wn,
                        int lane) const {
    stage_i8<Moe1I8, MI, NI, TM, TN, LDC>(*this, t, C, acc, wm, wn, lane);
  }
  // item = 8 expert units of one row (C holds silu(g) u)
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int CC = NC / 8;
    for (int it = tid; it < BM * CC; it += NT) {
      const int r = it / CC, c8 = (it % CC) * 8;
      if (r >= t.mvalid || t.n0 + c8 >= dff) continue;
      store8(h + int64_t(t.p0 + r) * dff + t.n0 + c8, C + r * LDC + c8);
    }
  }
};

struct Moe2I8 {
  typedef OpI8 Op;
  static constexpr int EPI = EPI_PLAIN;
  static constexpr bool GROUPED = true;
  const int8_t *a, *Wd;
  const float *sa, *sd;
  float *Y;  // rows in list order
  const int32_t *cnt;
  int E, d, pitch;
  static constexpr int out_cols(int BN) { return BN; }
  __device__ int tiles(int BM, int ny, const GroupScan &gs) const { return gs.total * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &gs) const {
    t.n0 = first_unit(by, BN);
    return mmap_grouped(bx, BM, gs, t);
  }
  __device__ static int first_unit(int by, int BN) { return by * BN; }
  __device__ const int8_t *a_row(const MTile &t, int r) const { return a + int64_t(t.p0 + r) * pitch; }
  __device__ const int8_t *b_row(const MTile &t, int n) const {
    return t.n0 + n < d ? Wd + (int64_t(t.e - 1) * d + t.n0 + n) * pitch : nullptr;
  }
  __device__ float row_scale(const MTile &t, int r) const { return sa[t.p0 + r]; }
  __device__ float col_scale(const MTile &t, int n) const {
    return t.n0 + n < d ? sd[int64_t(t.e - 1) * d + t.n0 + n] : 0.f;
  }
  // Four-wave kernel: columns as in LinearI8.
  static constexpr bool DIRECT_W4 = true;
  __device__ const int8_t *a_base() const { return a; }
  __device__ static int b_pick(int) { return 0; }
  template <int TN, int K>
  __device__ const int8_t *b_base_w4(int, int) const { return Wd; }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.p0 + r) * uint32_t(pitch); }
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int f = t.n0 + NI * (16 * wn + c) + ni;
    return f < d ? uint32_t((t.e - 1) * d + f) * uint32_t(pitch) : 0u;
  }
  __device__ const float *row_scale_at(const MTile &t, int r) const { return sa + t.p0 + r; }
  template <int TN>
  __device__ const float *col_scale_at(const MTile &t, int wn, int n) const {
    return sd + (int64_t(t.e - 1) * d + min(t.n0 + TN * wn + n, d - 1));
  }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const i32x4_t (&acc)[MI][NI], const float *scales, int wm,
                           int wn, int lane) const {
    static_assert(NI == 8, "whole 8-column pieces");
    const int f = t.n0 + NI * (16 * wn + (lane & 15));
    if (f >= d) return;  // d is a multiple of NI: a lane's columns are all in or all out
    float sc[NI];
    w4_cols<MI>(scales, lane, sc);
    float *out = Y + int64_t(t.p0) * d;  // (wave-uniform; a lane's offset fits 32 bits)
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int r0 = wm * MI * 16 + mi * 16 + 4 * (lane >> 4);
      const float4 sr = w4_rows<MI>(scales, mi, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) v[ni] = dequant(acc[mi][ni][i], elem(sr, i), sc[ni]);
        if (r0 + i < t.mvalid) store8(behind(out, uint32_t((r0 + i) * d + f) * 4u), v);
      }
    }
  }
  template <int MI, int NI, int TM, int TN, int LDC>
  __device__ void stage(const MTile &t, float *C, const i32x4_t (&acc)[MI][NI], int wm, int wn,
                        int lane) const {
    stage_i8<Moe2I8, MI, NI, TM, TN, LDC>(*this, t, C, acc, wm, wn, lane);
  }
  // item = 8 output features of one list row
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int CC = NC / 8;
    for (int it = tid; it < BM * CC; it += NT) {
      const int r = it / CC, c8 = (it % CC) * 8;
      if (r >= t.mvalid || t.n0 + c8 >= d) continue;
      store8(Y + int64_t(t.p0 + r) * d + t.n0 + c8, C + r * LDC + c8);
    }
  }
};

// ------------------------------------------------------------------ launchers
// Rows a launch may take: its blocks stay far below the limits of a grid, and (for the four-wave
// kernel's 32-bit offsets) its codes within 4 GB.
static int rows_a_launch(int c64, int pitch) {
  const int64_t near = ((int64_t(1) << 32) - 1) / pitch / 256 * 256;
  return int(std::min(int64_t(std::max(1, (1 << 22) / c64)) * 32, near));
}

// K groups of a block where there is one a CU at most: the chain of K steps is that much shorter, and
// sums of whole numbers may be split anywhere, evenly or not, so a token's result stays the same (300 x
// 8000 -> 100: 21.2 us, two groups 23.6, one 30.7; 64 x 8192 -> 4096: 21.2, two 23.4; QKV 64 x 2112:
// 10.9, 11.6, 12.8; 160M experts, 4 tokens: 22.9, two 23.5).
static int k_groups(int blocks, int K2) {
  return blocks > cu_count() || K2 < 128 ? 1 : K2 < 256 ? 2 : 4;
}
// 32 x 64 tiles
template <class P>
static hipError_t launch_32(const P &p, int K2, int m_tiles, int n_tiles, int blocks, hipStream_t st) {
  const int groups = k_groups(blocks, K2);
  if (groups == 4) return launch<P, 32, 64, 2, 1, 64, 3, 4>(p, K2, m_tiles, n_tiles, st);
  if (groups == 2) return launch<P, 32, 64, 2, 1, 64, 4, 2>(p, K2, m_tiles, n_tiles, st);
  return launch<P, 32, 64, 2, 1, 64, 4>(p, K2, m_tiles, n_tiles, st);
}

template <class P>
static hipError_t linear_rows(const P &all, hipStream_t st) {
  const int K2 = all.pitch / 2, c64 = (all.m + 63) / 64, c128 = (all.m + 127) / 128;
  const int most = rows_a_launch(c64, all.pitch);
  for (int at = 0; at < all.N; at += most) {
    P p = all;
    p.N = std::min(most, all.N - at);
    p.a += int64_t(at) * p.pitch;
    p.sa += at;
    p.y += at * p.ldy;
    if (p.res) p.res += at * p.ldr;
    hipError_t e = hipErrorInvalidValue;
    bool w4 = false;  // (rows of odd places are written from LDS by the smaller tiles)
    const int8_t *lo;
    const int m32 = (p.N + 31) / 32, m256 = (p.N + 255) / 256, c256 = (p.m + 255) / 256;
    if constexpr (P::WIDE)
      w4 = K2 >= 128 && span32({{p.a, size_t(p.N) * p.pitch}}, &lo) &&
           span32({{p.w, size_t(p.m) * p.pitch}}, &lo) &&
           std::max(p.ldy, p.ldr) < (1 << 22) && w4_rounds(p.N, c128, tile_cost(m256 * c256, COST_256X256));
    if (few_tiles(p.N, c128))
      e = launch_32(p, K2, m32, c64, m32 * c64, st);
    else if (!w4)
      e = launch_mid(p, K2, p.N, c128, st);
    else if constexpr (P::WIDE)
      e = launch_w4<P, 256, 256>(p, K2, m256, c256, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t i8_linear(int act, int N, int m, int k, const int8_t *a, const float *sa,
                     const triroute_i8_w &w, const void *res, int64_t ldr, void *y, int64_t ldy,
                     hipStream_t st) {
  auto run = [&](auto tag, auto vec) {
    using T = decltype(tag);
    LinearI8<T, decltype(vec)::value> p;
    p.a = a;
    p.sa = sa;
    p.w = (const int8_t *)w.codes;
    p.sw = w.scale;
    p.y = (T *)y;
    p.res = (const T *)res;
    p.ldy = ldy;
    p.ldr = ldr;
    p.N = N;
    p.m = m;
    p.pitch = i8_pitch(k);
    return linear_rows(p, st);
  };
  const int es = act == TRIROUTE_BF16 ? 2 : 4;
  const bool vec = m % 8 == 0 && ((uintptr_t(y) | uintptr_t(ldy * es)) & 15) == 0 &&
                   (!res || ((uintptr_t(res) | uintptr_t(ldr * es)) & 15) == 0);
  if (act == TRIROUTE_BF16) return vec ? run(bf16{}, std::true_type{}) : run(bf16{}, std::false_type{});
  return vec ? run(float{}, std::true_type{}) : run(float{}, std::false_type{});
}

hipError_t i8_qkv(const triroute_cfg &cfg, int N, const int8_t *a, const float *sa,
                  const triroute_dense_i8_w &w, const float *rope, void *q, void *k, void *v,
                  hipStream_t st) {
  auto run = [&](auto tag) {
    using T = decltype(tag);
    QkvI8<T> all;
    all.Wq = (const int8_t *)w.Wq.codes;
    all.Wk = (const int8_t *)w.Wk.codes;
    all.Wv = (const int8_t *)w.Wv.codes;
    all.sq = w.Wq.scale;
    all.sk = w.Wk.scale;
    all.sv = w.Wv.scale;
    all.pitch = i8_pitch(cfg.d_model);
    all.dh = cfg.head_dim;
    all.Hd = cfg.n_heads * cfg.head_dim;
    all.Kd = cfg.n_kv_heads * cfg.head_dim;
    all.Ncols = all.Hd + 2 * all.Kd;
    const int c64 = (all.Ncols + 63) / 64, most = rows_a_launch(c64, all.pitch), K2 = all.pitch / 2;
    for (int at = 0; at < N; at += most) {
      QkvI8<T> p = all;
      p.N = std::min(most, N - at);
      p.a = a + int64_t(at) * p.pitch;
      p.sa = sa + at;
      p.rope = (const float2 *)rope + int64_t(at) * (p.dh / 2);
      p.q = (T *)q + int64_t(at) * p.Hd;
      p.k = (T *)k + int64_t(at) * p.Kd;
      p.v = (T *)v + int64_t(at) * p.Kd;
      hipError_t e = hipErrorInvalidValue;
      const int8_t *lo;
      const int c128 = (p.Ncols + 127) / 128, m256 = (p.N + 255) / 256, c256 = (p.Ncols + 255) / 256;
      bool w4 = false;
      if constexpr (std::is_same<T, bf16>::value)
        w4 = K2 >= 128 && span32({{p.a, size_t(p.N) * p.pitch}}, &lo) &&
             span32({{p.Wq, size_t(p.Hd) * p.pitch}}, &lo) &&
             w4_rounds(p.N, c128, tile_cost(m256 * c256, COST_256X256));
      if (few_tiles(p.N, c128)) {
        const int m32 = (p.N + 31) / 32;
        if (p.dh == 64)
          e = launch_32(p, K2, m32, c64, m32 * c64, st);
        else if (k_groups(m32 * c64 / 2, K2) > 1)
          e = launch<QkvI8<T>, 32, 128, 2, 2, 64, 3, 2>(p, K2, m32, c64 / 2, st);
        else
          e = launch<QkvI8<T>, 32, 128, 2, 2, 64, 4>(p, K2, m32, c64 / 2, st);
      } else if (!w4) {
        e = launch_mid(p, K2, p.N, c128, st);
      } else if constexpr (std::is_same<T, bf16>::value) {
        e = launch_w4<QkvI8<T>, 256, 256>(p, K2, m256, c256, st);
      }
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  return cfg.act == TRIROUTE_BF16 ? run(bf16{}) : run(float{});
}

hipError_t i8_moe(const triroute_cfg &cfg, int N, const triroute_moe_i8_w &w,
                  const triroute_compaction &c, const MoeI8Ws &ws, hipStream_t st) {
  const int E = cfg.n_experts, Nk = N * cfg.top_k, d = cfg.d_model, dff = cfg.d_ff;
  // Rows of an expert when the router spreads its options evenly, and the tiles of BM rows that
  // the experts in use make then (a few rows more, as the counts vary).
  const int r = Nk / (E + 1);
  auto row_tiles = [&](int BM) { return std::min(E, Nk) * ((r + r / 32 + BM) / BM); };
  auto up = [&](auto f64) {
    typedef Moe1I8<decltype(f64)::value> P;
    P p;
    p.a = ws.n2;
    p.sa = ws.s_n2;
    p.Wg = (const int8_t *)w.Wgate.codes;
    p.Wu = (const int8_t *)w.Wup.codes;
    p.sg = w.Wgate.scale;
    p.su = w.Wup.scale;
    p.h = ws.h;
    p.cnt = c.exp_cnt;
    p.E = E;
    p.dff = dff;
    p.pitch = i8_pitch(d);
    const int K2 = p.pitch / 2;
    const size_t wb = size_t(E) * dff * p.pitch;
    const int8_t *lo;
    bool w4 = false;
    if constexpr (!decltype(f64)::value)
      w4 = r > 64 && K2 >= 128 && span32({{p.Wg, wb}}, &lo) &&
           span32({{p.a, size_t(Nk) * p.pitch}}, &lo) &&
           !one_round(row_tiles(128) * ((dff + 63) / 64));
    const int ny = (dff + 127) / 128;
    hipError_t e = hipErrorInvalidValue;
    const int c64 = (dff + 63) / 64;
    // Gate/up: as the bf16 product's rule (times of the two kernels measured alike), but 32-row tiles
    // with K groups where they leave CUs without a tile (160M, 1 token, two: 5.6 -> 5.1 us).
    const bool small = r <= 24 || (decltype(f64)::value && row_tiles(32) * ((dff + 31) / 32) <= 4 * cu_count());
    if (small) {
      const int c32 = (dff + 31) / 32;
      e = launch_32(p, K2, Nk / 32 + E, c32, row_tiles(32) * c32, st);
    } else if (r <= 64) {
      e = launch<P, 64, 128, 2, 2, 64, 3>(p, K2, Nk / 64 + E, c64, st);
    } else if (!w4) {
      e = launch<P, 128, 128, 4, 2, 64, 3>(p, K2, Nk / 128 + E, c64, st);
    } else if (row_tiles(128) * c64 <= 2 * cu_count()) {
      // one round, two blocks a CU (410M, 333 tokens, 352 tiles: the block 39.5 -> 38.0 us; 160M, 1150
      // tokens, 512: 52.4 -> 50.7; more tiles take longer here)
      e = launch<P, 128, 128, 2, 2, 64, 2>(p, K2, Nk / 128 + E, c64, st);
    } else if constexpr (!decltype(f64)::value) {
      if (tile_cost(row_tiles(128) * ny, 1.f) < tile_cost(row_tiles(256) * ny, 1.77f))
        e = launch_w4<P, 128, 256>(p, K2, Nk / 128 + E, ny, st);
      else
        e = launch_w4<P, 256, 256>(p, K2, Nk / 256 + E, ny, st);
    }
    if (e != hipSuccess) return e;
    return launch_i8_hidden(cfg, Nk, ws.h, c.exp_off, ws.hq, ws.s_h, st);
  };
  const hipError_t e = cfg.act == TRIROUTE_BF16 ? up(std::false_type{}) : up(std::true_type{});
  if (e != hipSuccess) return e;
  Moe2I8 p;
  p.a = ws.hq;
  p.sa = ws.s_h;
  p.Wd = (const int8_t *)w.Wdown.codes;
  p.sd = w.Wdown.scale;
  p.Y = ws.Y;
  p.cnt = c.exp_cnt;
  p.E = E;
  p.d = d;
  p.pitch = i8_pitch(dff);
  const int K2 = p.pitch / 2, c64 = (d + 63) / 64, c128 = (d + 127) / 128, c256 = (d + 255) / 256;
  const int8_t *lo;
  // Down.  Few columns and a long K: 32-row tiles up to two a CU, with K groups up to one (two: 160M, 1
  // token 8.0 -> 6.3 us, 410M, 64 tokens 10.2 -> 8.0; 410M, 333 tokens, 384 tiles: 12.4, 64-row
  // tiles 14.5; 1.3B, 32 tokens, 512: 34, 64-row tiles of two stages 44), then 64-row tiles (410M, 1000
  // tokens, 256 tiles: 17.1, 32-row 25.1, 128-row 19.4), from about 400 on the four-wave
  // kernel (1.3B, 1000 tokens, 512 tiles: 60, 64-row 72; 2500 tokens 97 and, of 256 rows, 90, 128-row
  // tiles 109).
  const int t32 = row_tiles(32) * c64;
  if (t32 <= 2 * cu_count()) return launch_32(p, K2, Nk / 32 + E, c64, t32, st);
  if (row_tiles(64) * c128 <= 400) return launch<Moe2I8, 64, 128, 2, 2, 64, 3>(p, K2, Nk / 64 + E, c128, st);
  if (K2 < 128 || !span32({{p.Wd, size_t(E) * d * p.pitch}}, &lo) ||
      !span32({{p.a, size_t(Nk) * p.pitch}}, &lo))
    return launch<Moe2I8, 128, 128, 4, 2, 64, 3>(p, K2, Nk / 128 + E, c128, st);
  if (row_tiles(256) > E && tile_cost(row_tiles(128) * c256, 1.f) < tile_cost(row_tiles(256) * c256, 1.77f))
    return launch_w4<Moe2I8, 128, 256>(p, K2, Nk / 128 + E, c256, st);
  return launch_w4<Moe2I8, 256, 256>(p, K2, Nk / 256 + E, c256, st);
}

}  // namespace tr
