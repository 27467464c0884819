// bf16 GEMMs of the layer on gfx950 MFMA: C = A B^T, both operands
// K-contiguous, fp32 accumulation (v_mfma_f32_16x16x32_bf16), on the kernels of
// gemm_kernels.hpp.
//
// Epilogues work on the accumulator registers.  Within a wave's 64 columns
// the B rows are ordered so that column j of 16-column block ni and block
// ni + 2 are partners: gate/up of one expert unit (SwiGLU), or RoPE pair
// (j, j + d_h/2) of one head.  Each lane therefore holds both partners.
//
//   QKV   : [n1] x [Wq;Wk;Wv]^T, rotate-half RoPE on q and k
//   O-proj: xt = x + o Wo^T
//   MoE-1 : H = silu(n2 Wgate_e^T) * (n2 Wup_e^T) per expert (paper Sec. 3.2 (B))
//   MoE-2 : Y = H Wdown_e^T
// n2, H and Y of the experts hold one row per entry of the expert lists, in
// list order (the lists lie back to back), so a tile's rows are contiguous.
#include "gemm_kernels.hpp"

namespace tr {

struct QkvM {
  typedef OpBf16 Op;
  static constexpr bool DIRECT_W4 = true;
  static constexpr int EPI = EPI_ROPE;
  const bf16 *n1, *Wq, *Wk, *Wv, *Wlo;  // Wlo: the lowest of Wq, Wk, Wv
  bf16 *q, *k, *v;
  const float2 *rope;  // (cos, sin) of token row, pair j at row * dh / 2 + j
  int N, d, H, Hkv, dh, Ncols;
  // four-wave kernel: byte offsets of Wq, Wk, Wv from Wlo less the first
  // column of their range times the row pitch, and the range ends
  uint32_t wq_o, wk_o, wv_o;
  int Hd, HKd;
  static constexpr int out_cols(int BN) { return BN; }
  static constexpr bool GROUPED = false;
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
  __device__ const bf16 *a_base() const { return n1; }
  __device__ const bf16 *b_base() const { return Wlo; }
  __device__ const bf16 *a_row(const MTile &t, int r) const { return n1 + int64_t(t.m0 + r) * d; }
  __device__ const bf16 *b_row(const MTile &t, int n) const {
    int P, half;
    col_pair(n, P, half);
    int gc = t.n0 + ccol(P, half);
    if (gc >= Ncols) return nullptr;
    const int Hd = H * dh, Kd = Hkv * dh;
    if (gc < Hd) return Wq + int64_t(gc) * d;
    gc -= Hd;
    if (gc < Kd) return Wk + int64_t(gc) * d;
    return Wv + int64_t(gc - Kd) * d;
  }
  // Four-wave kernel (128-column tiles, d_h 64 or 128): wave column wn
  // holds pairs j = jw + 2 c + (ni >> 1) of one head, the first half of the
  // pair in block ni even and the second (j + d_h / 2) in ni odd, where
  // d_h 64: the tile's head wn, jw = 0; d_h 128: the tile's one head, jw = 32 wn.
  // Each lane thus holds both halves of pairs 2 c, 2 c + 1 of its rows.
  __device__ void w4_head(const MTile &t, int wn, int &hcol, int &jw) const {
    hcol = t.n0 + (dh == 64 ? 64 * wn : 0);  // first column of the head
    jw = dh == 64 ? 0 : 32 * wn;
  }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.m0 + r) * uint32_t(2 * d); }
  // 256-column tiles (d_h 128 only): wave column wn holds the tile's head
  // wn, lane column c pairs j = 4 c + (ni >> 1), first halves in even ni.
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    int hcol, jw;
    if constexpr (NI == 8) {
      hcol = t.n0 + 128 * wn;
      jw = 0;
    } else {
      w4_head(t, wn, hcol, jw);
    }
    const int gc = hcol + jw + (NI / 2) * c + (ni >> 1) + (ni & 1) * (dh >> 1);
    // (arithmetic on the field values: a select of fields by a lane-varying
    // condition becomes a per-lane load from the kernel arguments)
    const uint32_t base = wq_o + uint32_t(gc >= Hd) * (wk_o - wq_o) + uint32_t(gc >= HKd) * (wv_o - wk_o);
    return gc < Ncols ? base + uint32_t(gc) * uint32_t(2 * d) : 0u;
  }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn, int lane) const {
    if constexpr (NI == 8)
      store_w4_wide(t, acc, wm, wn, lane);
    else
      store_w4_narrow(t, acc, wm, wn, lane);
  }
  // 256-column tiles: each lane holds both halves of pairs j .. j + 3 of
  // head wn; the rotation entries of a row block mi are loaded one block
  // ahead of their use.
  template <int MI, int NI>
  __device__ void store_w4_wide(const MTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn,
                                int lane) const {
    const int hcol = t.n0 + 128 * wn;
    if (hcol >= Ncols) return;
    const int Hd = H * dh, Kd = Hkv * dh, hd = dh >> 1;
    bf16 *out = q;
    int ld = Hd, col = hcol;
    bool rot = true;
    if (hcol >= Hd + Kd) {
      out = v; ld = Kd; col = hcol - Hd - Kd; rot = false;
    } else if (hcol >= Hd) {
      out = k; ld = Kd; col = hcol - Hd;
    }
    const int j = 4 * (lane & 15);
    auto row_of = [&](int mi, int i) { return wm * MI * 16 + mi * 16 + 4 * (lane >> 4) + i; };
    auto load_cs = [&](int mi, float4 (&cs)[4][2]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = row_of(mi, i);
        const float4 *tb = (const float4 *)(rope + int64_t(t.m0 + (r < t.mvalid ? r : 0)) * hd + j);
        cs[i][0] = tb[0];
        cs[i][1] = tb[1];
      }
    };
    float4 cur[4][2], nxt[4][2];
    if (rot) load_cs(0, cur);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      if (rot && mi + 1 < MI) load_cs(mi + 1, nxt);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = row_of(mi, i);
        float y1[4], y2[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float a1 = acc[mi][2 * u][i], a2 = acc[mi][2 * u + 1][i];
          y1[u] = a1;
          y2[u] = a2;
          if (rot) {
            const float4 c4 = cur[i][u >> 1];  // (cos, sin) of pairs j + 2 (u / 2), + 1
            const float cs = (u & 1) ? c4.z : c4.x, sn = (u & 1) ? c4.w : c4.y;
            y1[u] = a1 * cs - a2 * sn;
            y2[u] = a1 * sn + a2 * cs;
          }
        }
        if (r < t.mvalid) {
          bf16 *o = out + int64_t(t.m0 + r) * ld + col + j;
          *(uint2 *)o = make_uint2(pk_bf16(y1[0], y1[1]), pk_bf16(y1[2], y1[3]));
          *(uint2 *)(o + hd) = make_uint2(pk_bf16(y2[0], y2[1]), pk_bf16(y2[2], y2[3]));
        }
      }
      if (rot && mi + 1 < MI) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          cur[i][0] = nxt[i][0];
          cur[i][1] = nxt[i][1];
        }
      }
    }
  }
  template <int MI, int NI>
  __device__ void store_w4_narrow(const MTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn,
                                  int lane) const {
    static_assert(NI == 4, "two pairs per lane");
    int hcol, jw;
    w4_head(t, wn, hcol, jw);
    if (hcol >= Ncols) return;
    const int Hd = H * dh, Kd = Hkv * dh, hd = dh >> 1;
    bf16 *out = q;
    int ld = Hd, col = hcol;
    bool rot = true;
    if (hcol >= Hd + Kd) {
      out = v; ld = Kd; col = hcol - Hd - Kd; rot = false;
    } else if (hcol >= Hd) {
      out = k; ld = Kd; col = hcol - Hd;
    }
    const int j = jw + 2 * (lane & 15);
    // the rows' rotation entries first, so their loads overlap
    float4 cs[MI][4];
    if (rot) {
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = wm * MI * 16 + mi * 16 + 4 * (lane >> 4) + i;
          cs[mi][i] = *(const float4 *)(rope + int64_t(t.m0 + (r < t.mvalid ? r : 0)) * hd + j);
        }
    }
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = wm * MI * 16 + mi * 16 + 4 * (lane >> 4) + i;
        if (r >= t.mvalid) continue;
        const float a10 = acc[mi][0][i], a20 = acc[mi][1][i], a11 = acc[mi][2][i], a21 = acc[mi][3][i];
        float y10 = a10, y20 = a20, y11 = a11, y21 = a21;
        if (rot) {
          const float4 c4 = cs[mi][i];  // (cos, sin) of pairs j and j + 1
          y10 = a10 * c4.x - a20 * c4.y;
          y20 = a10 * c4.y + a20 * c4.x;
          y11 = a11 * c4.z - a21 * c4.w;
          y21 = a11 * c4.w + a21 * c4.z;
        }
        bf16 *o = out + int64_t(t.m0 + r) * ld + col + j;
        *(uint32_t *)o = pk_bf16(y10, y11);
        *(uint32_t *)(o + hd) = pk_bf16(y20, y21);
      }
  }
  // item = (row, 8 consecutive pairs of one head): rotate-half RoPE on q and
  // k from the token's rotation table; v is copied.
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int PC = NC / 16;  // 8-pair chunks per row
    const int Hd = H * dh, Kd = Hkv * dh, hd = dh >> 1;
    for (int it = tid; it < BM * PC; it += NT) {
      const int r = it / PC, P0 = (it % PC) * 8;
      const int lc1 = (P0 / hd) * dh + (P0 % hd);
      const int c1 = t.n0 + lc1;
      if (r >= t.mvalid || c1 >= Ncols) continue;
      const int row = t.m0 + r;
      bf16 *out;
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
        const float4 *tb = (const float4 *)(rope + int64_t(row) * hd + col % hd);
#pragma unroll
        for (int u2 = 0; u2 < 4; ++u2) {
          const float4 cs2 = tb[u2];  // pairs 2 u2 and 2 u2 + 1
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int u = 2 * u2 + h;
            const float cs = h ? cs2.z : cs2.x, sn = h ? cs2.w : cs2.y;
            const float a1 = y1[u], a2 = y2[u];
            y1[u] = a1 * cs - a2 * sn;
            y2[u] = a1 * sn + a2 * cs;
          }
        }
      }
      bf16 *o = out + int64_t(row) * ld + col;
      *(u32x4_t *)o = pack8_bf16(y1);
      *(u32x4_t *)(o + hd) = pack8_bf16(y2);
    }
  }
};

struct OprojM {
  typedef OpBf16 Op;
  static constexpr bool DIRECT_W4 = true;
  static constexpr int EPI = EPI_PLAIN;
  const bf16 *o, *Wo, *x;
  bf16 *xt;
  int N, d, K;
  static constexpr int out_cols(int BN) { return BN; }
  static constexpr bool GROUPED = false;
  __device__ int tiles(int BM, int ny, const GroupScan &) const { return (N + BM - 1) / BM * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &) const {
    t.m0 = bx * BM;
    t.n0 = by * BN;
    t.mvalid = min(BM, N - t.m0);
    t.e = t.p0 = 0;
    return t.mvalid > 0;
  }
  __device__ const bf16 *a_base() const { return o; }
  __device__ const bf16 *b_base() const { return Wo; }
  __device__ const bf16 *a_row(const MTile &t, int r) const { return o + int64_t(t.m0 + r) * K; }
  __device__ const bf16 *b_row(const MTile &t, int n) const {
    return t.n0 + n < d ? Wo + int64_t(t.n0 + n) * K : nullptr;
  }
  // Four-wave kernel: in wave column wn, MFMA block ni, lane column c holds
  // output column NI (16 wn + c) + ni of the tile, so each lane ends with NI
  // consecutive columns of each of its rows: xt = x + o Wo^T in pieces of
  // NI / 2 words.
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int f = t.n0 + NI * (16 * wn + c) + ni;
    return f < d ? uint32_t(f) * uint32_t(2 * K) : 0u;
  }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.m0 + r) * uint32_t(2 * K); }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn, int lane) const {
    static_assert(NI % 2 == 0, "whole words");
    const int f = t.n0 + NI * (16 * wn + (lane & 15));
    if (f >= d) return;  // d is a multiple of NI: a lane's columns are all in or all out
    // in halves of the rows (MI / 2 row blocks): each half's residual rows
    // are loaded first, so their loads overlap (all at once would hold 4 MI
    // (NI / 2) registers)
    constexpr int MH = MI / 2;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t xv[MH][4][NI / 2];
#pragma unroll
      for (int m = 0; m < MH; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = wm * MI * 16 + (h * MH + m) * 16 + 4 * (lane >> 4) + i;
          const uint32_t *xr = (const uint32_t *)(x + int64_t(t.m0 + (r < t.mvalid ? r : 0)) * d + f);
#pragma unroll
          for (int u = 0; u < NI / 2; ++u) xv[m][i][u] = xr[u];
        }
#pragma unroll
      for (int m = 0; m < MH; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int mi = h * MH + m;
          const int r = wm * MI * 16 + mi * 16 + 4 * (lane >> 4) + i;
          if (r >= t.mvalid) continue;
          uint32_t *yr = (uint32_t *)(xt + int64_t(t.m0 + r) * d + f);
#pragma unroll
          for (int u = 0; u < NI / 2; ++u) {
            const uint32_t w = xv[m][i][u];
            yr[u] = pk_bf16(__uint_as_float(w << 16) + acc[mi][2 * u][i],
                            __uint_as_float(w & 0xFFFF0000u) + acc[mi][2 * u + 1][i]);
          }
        }
    }
  }
  // item = 8 columns of one row: xt = x + o Wo^T
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int CC = NC / 8;
    for (int it = tid; it < BM * CC; it += NT) {
      const int r = it / CC, c8 = (it % CC) * 8;
      if (r >= t.mvalid || t.n0 + c8 >= d) continue;
      const int64_t off = int64_t(t.m0 + r) * d + t.n0 + c8;
      const u32x4_t xv = *(const u32x4_t *)(x + off);
      float y[8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        y[2 * u] = __uint_as_float(xv[u] << 16) + C[r * LDC + c8 + 2 * u];
        y[2 * u + 1] = __uint_as_float(xv[u] & 0xFFFF0000u) + C[r * LDC + c8 + 2 * u + 1];
      }
      *(u32x4_t *)(xt + off) = pack8_bf16(y);
    }
  }
};

struct Moe1M {
  typedef OpBf16 Op;
  static constexpr int EPI = EPI_SWIGLU;
  const bf16 *n2, *Wg, *Wu, *Wlo;  // n2: normalised rows in list order; Wlo: the lower of Wg, Wu
  bf16 *Hm;
  const int32_t *cnt;
  int E, d, dff;
  static constexpr int out_cols(int BN) { return BN / 2; }
  static constexpr bool GROUPED = true;
  __device__ int tiles(int BM, int ny, const GroupScan &gs) const { return gs.total * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &gs) const {
    if (!mmap_grouped(bx, BM, gs, t)) return false;
    t.n0 = by * (BN / 2);  // BN/2 expert units per tile (gate + up columns)
    return true;
  }
  __device__ int ccol(int P, int) const { return P; }
  __device__ const bf16 *a_base() const { return n2; }
  __device__ const bf16 *b_base() const { return Wlo; }
  __device__ const bf16 *a_row(const MTile &t, int r) const { return n2 + int64_t(t.p0 + r) * d; }
  __device__ const bf16 *b_row(const MTile &t, int n) const {
    int P, half;
    col_pair(n, P, half);
    const int f = t.n0 + P;
    if (f >= dff) return nullptr;
    return (half ? Wu : Wg) + (int64_t(t.e - 1) * dff + f) * d;
  }
  // Four-wave kernel: in wave column wn, MFMA block ni, lane column c
  // holds expert unit (NI / 2) (16 wn + c) + ni / 2 of the tile, gate for
  // even ni and up for odd, so each lane ends with both halves of NI / 2
  // consecutive units and writes them as one piece per row.
  static constexpr bool DIRECT_W4 = true;
  // Byte offsets from a_base / b_base (32 bits: the host checks the spans).
  // Units past d_ff read unit 0 of the lower matrix instead.
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.p0 + r) * uint32_t(2 * d); }
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int f = t.n0 + (NI / 2) * (16 * wn + c) + (ni >> 1);
    if (f >= dff) return 0u;
    const uint32_t m = uint32_t(((ni & 1) ? Wu : Wg) - Wlo) * 2u;
    return m + uint32_t((t.e - 1) * dff + f) * uint32_t(2 * d);
  }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn, int lane) const {
    static_assert(NI == 8, "4 units per lane, one 8-byte piece per row");
    const int f = t.n0 + (NI / 2) * (16 * wn + (lane & 15));
    if (f >= dff) return;  // d_ff is a multiple of 4: a lane's units are all in or all out
    // SwiGLU of every value first (independent chains for the VALU to
    // overlap), then the stores of the valid rows
    uint32_t w[MI][4][2];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float g0 = acc[mi][4 * u][i], u0 = acc[mi][4 * u + 1][i];
          const float g1 = acc[mi][4 * u + 2][i], u1 = acc[mi][4 * u + 3][i];
          w[mi][i][u] = pk_bf16(g0 * __builtin_amdgcn_rcpf(1.0f + __expf(-g0)) * u0,
                                g1 * __builtin_amdgcn_rcpf(1.0f + __expf(-g1)) * u1);
        }
    bf16 *out = Hm + int64_t(t.p0) * dff + f;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = wm * MI * 16 + mi * 16 + 4 * (lane >> 4) + i;
        if (r < t.mvalid) *(uint2 *)(out + r * dff) = make_uint2(w[mi][i][0], w[mi][i][1]);
      }
  }
  // item = 8 expert units of one assignment row (C holds silu(g) u)
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int CC = NC / 8;
    for (int it = tid; it < BM * CC; it += NT) {
      const int r = it / CC, c8 = (it % CC) * 8;
      if (r >= t.mvalid || t.n0 + c8 >= dff) continue;
      *(u32x4_t *)(Hm + int64_t(t.p0 + r) * dff + t.n0 + c8) = pack8_bf16(C + r * LDC + c8);
    }
  }
};

struct Moe2M {
  typedef OpBf16 Op;
  static constexpr bool DIRECT_W4 = true;
  static constexpr int EPI = EPI_PLAIN;
  const bf16 *Hm, *Wd;
  float *Y;  // rows in list order
  const int32_t *cnt;
  int E, d, dff;
  int ksplit = 1;        // K halves (few-token path), each to its own plane of Y
  int64_t yplane = 0;    // elements between planes
  static constexpr int out_cols(int BN) { return BN; }
  static constexpr bool GROUPED = true;
  __device__ int tiles(int BM, int ny, const GroupScan &gs) const { return gs.total * ny; }
  __device__ bool map(int bx, int by, int BM, int BN, MTile &t, const GroupScan &gs) const {
    if (!mmap_grouped(bx, BM, gs, t)) return false;
    const int ncol = (d + BN - 1) / BN, kh = by / ncol;
    t.n0 = (by - kh * ncol) * BN;
    t.k0 = kh * (dff / ksplit);
    t.yp = kh;
    return true;
  }
  __device__ const bf16 *a_base() const { return Hm; }
  __device__ const bf16 *b_base() const { return Wd; }
  __device__ const bf16 *a_row(const MTile &t, int r) const {
    return Hm + int64_t(t.p0 + r) * dff + t.k0;
  }
  __device__ const bf16 *b_row(const MTile &t, int n) const {
    return t.n0 + n < d ? Wd + (int64_t(t.e - 1) * d + t.n0 + n) * dff + t.k0 : nullptr;
  }
  // Four-wave kernel: in wave column wn, MFMA block ni, lane column c
  // holds output feature NI (16 wn + c) + ni of the tile, so each lane ends
  // with NI consecutive features of each of its rows.
  template <int NI>
  __device__ uint32_t b_off_w4(const MTile &t, int wn, int ni, int c) const {
    const int f = t.n0 + NI * (16 * wn + c) + ni;
    return f < d ? uint32_t((t.e - 1) * d + f) * uint32_t(2 * dff) : 0u;
  }
  __device__ uint32_t a_off(const MTile &t, int r) const { return uint32_t(t.p0 + r) * uint32_t(2 * dff); }
  template <int MI, int NI>
  __device__ void store_w4(const MTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn, int lane) const {
    static_assert(NI % 2 == 0, "whole 8-byte pieces");
    const int f = t.n0 + NI * (16 * wn + (lane & 15));
    if (f >= d) return;  // d is a multiple of NI: a lane's features are all in or all out
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = wm * MI * 16 + mi * 16 + 4 * (lane >> 4) + i;
        if (r >= t.mvalid) continue;
        float *y = Y + int64_t(t.p0 + r) * d + f;
#pragma unroll
        for (int ni = 0; ni < NI; ni += 2) *(float2 *)(y + ni) = make_float2(acc[mi][ni][i], acc[mi][ni + 1][i]);
      }
  }
  // item = 8 output features of one list row
  template <int BM, int NC, int LDC, int NT>
  __device__ void epilogue(const MTile &t, const float *C, int tid) const {
    constexpr int CC = NC / 8;
    for (int it = tid; it < BM * CC; it += NT) {
      const int r = it / CC, c8 = (it % CC) * 8;
      if (r >= t.mvalid || t.n0 + c8 >= d) continue;
      float *y = Y + t.yp * yplane + int64_t(t.p0 + r) * d + t.n0 + c8;
      const float *c = C + r * LDC + c8;
      *(float4 *)y = make_float4(c[0], c[1], c[2], c[3]);
      *(float4 *)(y + 4) = make_float4(c[4], c[5], c[6], c[7]);
    }
  }
};


// ------------------------------------------------------------------ launchers
hipError_t mfma_qkv(const triroute_cfg &cfg, int B, int Tq, const void *n1,
                    const triroute_dense_w &w, const float *rope, void *q, void *k, void *v,
                    hipStream_t st) {
  QkvM p;
  p.n1 = (const bf16 *)n1;
  p.Wq = (const bf16 *)w.Wq;
  p.Wk = (const bf16 *)w.Wk;
  p.Wv = (const bf16 *)w.Wv;
  p.Wlo = std::min(p.Wq, std::min(p.Wk, p.Wv));
  p.q = (bf16 *)q;
  p.k = (bf16 *)k;
  p.v = (bf16 *)v;
  p.rope = (const float2 *)rope;
  p.N = B * Tq;
  p.d = cfg.d_model;
  p.H = cfg.n_heads;
  p.Hkv = cfg.n_kv_heads;
  p.dh = cfg.head_dim;
  p.Ncols = (cfg.n_heads + 2 * cfg.n_kv_heads) * cfg.head_dim;
  const int c128 = (p.Ncols + 127) / 128;
  // Few tokens (decode): the product streams the weights; 32-row tiles one
  // head wide put one block on every head and row tile.  (Two K groups a
  // block would take 1.5 us off 9.3 on the 410M layer, but keys and values go
  // into the cache, and every other tile here sums them in one order of K: for
  // the same x a token's stored codes do not depend on how many tokens came
  // with it.  Behind a layer they may: the O-projection and the experts pick
  // tiles by the token count, and K groups or halves change the last bits of
  // the x_out that the next layer stores keys and values of.)
  if (few_tiles(p.N, c128)) {
    if (p.dh == 64)
      return launch<QkvM, 32, 64, 2, 1, 64, 4>(p, cfg.d_model, (p.N + 31) / 32, (p.Ncols + 63) / 64, st);
    return launch<QkvM, 32, 128, 2, 2, 64, 4>(p, cfg.d_model, (p.N + 31) / 32, c128, st);
  }
  const bf16 *lo;
  const bool w4 = p.Ncols % 128 == 0 && p.d >= 128 &&
                  span32({{p.Wq, size_t(p.H) * p.dh * p.d * sizeof(bf16)},
                          {p.Wk, size_t(p.Hkv) * p.dh * p.d * sizeof(bf16)},
                          {p.Wv, size_t(p.Hkv) * p.dh * p.d * sizeof(bf16)}}, &lo) &&
                  span32({{p.n1, size_t(p.N) * p.d * sizeof(bf16)}}, &lo);
  // d_h 128: one head per wave column on 256-column tiles (long K steps),
  // where the columns divide into them
  const bool wide = p.dh == 128 && p.Ncols % 256 == 0;
  const int mt = (p.N + 255) / 256;
  if (w4 && w4_rounds(p.N, c128, wide ? tile_cost(mt * (p.Ncols / 256), COST_256X256)
                                      : tile_cost(mt * c128, COST_256X128))) {
    const uint32_t pitch = 2u * uint32_t(p.d);
    p.Hd = p.H * p.dh;
    p.HKd = p.Hd + p.Hkv * p.dh;
    p.wq_o = uint32_t((const uint8_t *)p.Wq - (const uint8_t *)p.Wlo);
    p.wk_o = uint32_t((const uint8_t *)p.Wk - (const uint8_t *)p.Wlo) - uint32_t(p.Hd) * pitch;
    p.wv_o = uint32_t((const uint8_t *)p.Wv - (const uint8_t *)p.Wlo) - uint32_t(p.HKd) * pitch;
    if (wide) return launch_w4<QkvM, 256, 256>(p, cfg.d_model, mt, p.Ncols / 256, st);
    return launch_w4<QkvM, 256, 128>(p, cfg.d_model, mt, c128, st);
  }
  return launch_mid(p, cfg.d_model, p.N, c128, st);
}

hipError_t mfma_oproj(const triroute_cfg &cfg, int N, const void *x, const void *o,
                      const triroute_dense_w &w, void *xt, hipStream_t st) {
  OprojM p;
  p.o = (const bf16 *)o;
  p.Wo = (const bf16 *)w.Wo;
  p.x = (const bf16 *)x;
  p.xt = (bf16 *)xt;
  p.N = N;
  p.d = cfg.d_model;
  p.K = cfg.n_heads * cfg.head_dim;
  const int c128 = (p.d + 127) / 128;
  if (few_tiles(N, c128) && split_k((N + 31) / 32 * ((p.d + 63) / 64), p.K))
    return launch<OprojM, 32, 64, 2, 1, 64, 4, 2>(p, p.K, (N + 31) / 32, (p.d + 63) / 64, st);
  if (few_tiles(N, c128))  // few tokens: weight streaming, narrow tiles as for QKV
    return launch<OprojM, 32, 64, 2, 1, 64, 4>(p, p.K, (N + 31) / 32, (p.d + 63) / 64, st);
  const bf16 *lo;
  const bool w4 = p.K >= 128 && span32({{p.o, size_t(N) * p.K * sizeof(bf16)}}, &lo) &&
                  span32({{p.Wo, size_t(p.d) * p.K * sizeof(bf16)}}, &lo);
  if (w4) {
    const int mt = (N + 255) / 256;
    const float t192 = p.d % 192 == 0 ? tile_cost(mt * (p.d / 192), COST_256X192) : 1e30f;
    const float t256 = p.d % 256 == 0 ? tile_cost(mt * (p.d / 256), COST_256X256) : 1e30f;
    if (w4_rounds(N, c128, std::min(t192, t256))) {
      if (t192 <= t256) return launch_w4<OprojM, 256, 192>(p, p.K, mt, p.d / 192, st);
      return launch_w4<OprojM, 256, 256>(p, p.K, mt, p.d / 256, st);
    }
  }
  return launch_mid(p, p.K, N, c128, st);
}

hipError_t mfma_moe(const triroute_cfg &cfg, int N, const void *n2, const triroute_moe_w &w,
                    const triroute_compaction &c, void *Hm, float *Y, hipStream_t st) {
  const int E = cfg.n_experts, k = cfg.top_k, d = cfg.d_model, dff = cfg.d_ff;
  const int Nk = N * k;
  Moe1M p1;
  p1.n2 = (const bf16 *)n2;
  p1.Wg = (const bf16 *)w.Wgate;
  p1.Wu = (const bf16 *)w.Wup;
  p1.Hm = (bf16 *)Hm;
  p1.cnt = c.exp_cnt;
  p1.E = E;
  p1.d = d;
  p1.dff = dff;
  const size_t wb = size_t(E) * dff * d * sizeof(bf16);
  const bf16 *alo;
  // Rows an expert has when the router spreads its options evenly, and the
  // tiles of BM rows that E such experts make (a few rows more, as the
  // counts vary).
  const int r = Nk / (E + 1);
  auto row_tiles = [&](int BM) { return E * ((r + r / 32 + BM) / BM); };
  // Gate/up.  Up to 24 rows an expert the work is streaming the expert
  // weights: narrow 32 x 64 tiles (two waves, four stages) put every CU on
  // its own slice of them.  Up to 64 rows one 64-row tile reads each weight
  // once (the 32-row tiles read it per row tile).  Above, 128 x 128 tiles if
  // they make one round, else the four-wave kernel with 128- or 256-row
  // tiles, whichever needs less time for its rounds (a 256-row tile takes
  // 1.77 times a 128-row one).  Gate/up alone within the expert block (us;
  // weights not in a cache; before: 32-row tiles up to 2048 assignments,
  // 256-row tiles above): the block on 410M at 200 tokens 57 -> 49, 400
  // 82 -> 62, 700 118 -> 82, 2000 136 -> 133; 1.3B 400 402 -> 282, 700
  // 598 -> 351, 1000 789 -> 419; 160M 400 53 -> 40, 700 72 -> 53.
  const bool w4 = d >= 128 && span32({{p1.Wg, wb}, {p1.Wu, wb}}, &p1.Wlo) &&
                  span32({{p1.n2, size_t(Nk) * d * sizeof(bf16)}}, &alo);
  const int ny = (dff + 127) / 128;
  hipError_t err;
  if (r <= 24 && d >= 2048 && d % 128 == 0)
    // a long K: two K groups of three stages have more of the weights in
    // flight (1.3B, 32 to 100 tokens: the block 204 to 213 -> 193 to 202 us;
    // 410M, K 1024: 40 -> 43; nothing between the two was measured)
    err = launch<Moe1M, 32, 64, 2, 1, 64, 3, 2>(p1, d, Nk / 32 + E, (dff + 31) / 32, st);
  else if (r <= 24)
    err = launch<Moe1M, 32, 64, 2, 1, 64, 4>(p1, d, Nk / 32 + E, (dff + 31) / 32, st);
  else if (r <= 64)
    err = launch<Moe1M, 64, 128, 2, 2, 64, 3>(p1, d, Nk / 64 + E, (dff + 63) / 64, st);
  else if (!w4 || one_round(row_tiles(128) * ((dff + 63) / 64)))
    err = launch<Moe1M, 128, 128, 4, 2, 64, 3>(p1, d, Nk / 128 + E, (dff + 63) / 64, st);
  else if (tile_cost(row_tiles(128) * ny, 1.f) < tile_cost(row_tiles(256) * ny, 1.77f))
    err = launch_w4<Moe1M, 128, 256>(p1, d, Nk / 128 + E, ny, st);
  else
    err = launch_w4<Moe1M, 256, 256>(p1, d, Nk / 256 + E, ny, st);
  if (err != hipSuccess) return err;
  Moe2M p2;
  p2.Hm = (const bf16 *)Hm;
  p2.Wd = (const bf16 *)w.Wdown;
  p2.Y = Y;
  p2.cnt = c.exp_cnt;
  p2.E = E;
  p2.d = d;
  p2.dff = dff;
  // Down.  Up to 2048 assignments K is split in halves, each with its plane
  // of Y (moe_ysplit); 64- or 128-row tiles where they fill the CUs or the
  // rows fill them, else the 32-row tiles (down alone within the block, us:
  // 1.3B 400 tokens 402 -> 361, 700 598 -> 508; 410M 400 82 -> 75, 1000 154 -> 135;
  // 410M 100, 16 rows an expert: 32-row tiles 41.5, 64-row 45.8).
  const int c128 = (d + 127) / 128;
  if (Nk <= 2048) {
    p2.ksplit = moe_ysplit(cfg, N);
    p2.yplane = int64_t(Nk) * d;
    const int K = dff / p2.ksplit, cols = c128 * p2.ksplit;
    if (r > 64 && row_tiles(128) * cols >= 256)
      return launch<Moe2M, 128, 128, 4, 2, 64, 3>(p2, K, Nk / 128 + E, cols, st);
    if (r > 64) return launch<Moe2M, 64, 128, 2, 2, 64, 3>(p2, K, Nk / 64 + E, cols, st);
    // (with fewer assignments than experts not every expert has a tile: 32 x 64
    // tiles, two K groups a block; 1.3B, 1 token: the block 50 -> 35 us, 4 108 -> 96)
    if (Nk <= E && K % 128 == 0 && (K >= 2048 || Nk * 2 * cols <= 128))
      return launch<Moe2M, 32, 64, 2, 1, 64, 4, 2>(p2, K, Nk / 32 + E, (d + 63) / 64 * p2.ksplit, st);
    if (row_tiles(64) * cols >= 256)
      return launch<Moe2M, 64, 128, 2, 2, 64, 2>(p2, K, Nk / 64 + E, cols, st);
    return launch<Moe2M, 32, 64, 2, 1, 64, 4>(p2, K, Nk / 32 + E, (d + 63) / 64 * p2.ksplit, st);
  }
  // Above: 128 x 128 tiles if they make one round (410M, 2000 tokens: the
  // block 136 -> 106 us), else the four-wave kernel, with 256-row tiles where
  // one holds an expert's rows (each weight is read once: 1.3B, 2000 tokens,
  // 360 us, 128-row tiles 371) or their rounds are cheaper (192-wide ones
  // where they divide d), else 128-row ones (410M, 3000 tokens: 165 -> 150).
  const bool w4b = dff >= 128 && (d % 192 == 0 || d % 256 == 0) && span32({{p2.Wd, wb}}, &alo) &&
                   span32({{p2.Hm, size_t(Nk) * dff * sizeof(bf16)}}, &alo);
  if (!w4b || one_round(row_tiles(128) * c128))
    return launch<Moe2M, 128, 128, 4, 2, 64, 3>(p2, dff, Nk / 128 + E, c128, st);
  const bool by192 = d % 192 == 0;
  const float t128 = tile_cost(row_tiles(128) * (d / 256), 1.f);
  const float t256 = tile_cost(row_tiles(256) * (by192 ? d / 192 : d / 256), by192 ? 1.5f : 1.77f);
  if (d % 256 == 0 && row_tiles(256) > E && t128 < t256)
    return launch_w4<Moe2M, 128, 256>(p2, dff, Nk / 128 + E, d / 256, st);
  if (by192) return launch_w4<Moe2M, 256, 192>(p2, dff, Nk / 256 + E, d / 192, st);
  return launch_w4<Moe2M, 256, 256>(p2, dff, Nk / 256 + E, d / 256, st);
}

}  // namespace tr
