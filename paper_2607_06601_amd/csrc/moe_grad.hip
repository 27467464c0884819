// Backward pass of the experts' gated feed-forward block (paper Sec. 3.2 (B),
// second half of the Sec. 3.1 block).  Per assignment of a token to expert e
// with gate p (n the normalised row, dx the gradient of x_out):
//   G = Wg n, U = Wu n, q = Wd^T dx, s = 1 / (1 + exp(-G))
//   g_gate = <q, s G U>;  dU = p q s G;  dG = p q U s (1 + G (1 - s))
//   dWd += dx (p s G U)^T, dWg += dG n^T, dWu += dU n^T
//   dn += Wg^T dG + Wu^T dU
// and through the norm to xt and g2.  Three grouped products:
//   hidden  [G; U; q] of a tile of units and rows, whose sum indices are all d_model,
//           so that one epilogue holds the three in fp32 and g_gate is summed from
//           values that were not rounded (many rows: q comes from a product of its own,
//           in fp32, and the epilogue of G and U reads it)
//   input   dn = [dG dU] [Wg; Wu]
//   weight  dWg, dWu, dWd: sums over the rows of an expert
// Rows lie by expert, each expert's padded to a multiple of 64 rows with zeros: a
// padded row adds nothing to the weight gradients, so their K steps are whole.
// Operands whose sum index is not their contiguous one (Wd in hidden, Wg and
// Wu in input, both sides of weight) are staged as they lie, K rows of
// columns, and read as fragments by the transposing LDS load
// (ds_read_b64_tr_b16), so no transposed copy is made.
#include <type_traits>
#include <utility>

#include "gemm_tile.hpp"
#include "kernels.hpp"

namespace tr {

// ------------------------------------------------------------------ row maps
// Lane e - 1 of every wave holds expert e: rows, padded rows, and the sums before it.
struct PadScan {
  int c, pc;         // rows, padded rows
  int list, pad;     // first list entry, first padded row
  int total;         // all padded rows
};
__device__ __forceinline__ PadScan pad_scan(const int32_t *cnt, int E) {
  const int lane = threadIdx.x & 63;
  PadScan g;
  g.c = lane < E ? cnt[lane + 1] : 0;
  g.pc = (g.c + MOE_PAD - 1) / MOE_PAD * MOE_PAD;
  int a = g.c, b = g.pc;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(a, d, 64), y = __shfl_up(b, d, 64);
    if (lane >= d) {
      a += x;
      b += y;
    }
  }
  g.list = a - g.c;
  g.pad = b - g.pc;
  g.total = __shfl(b, 63, 64);
  return g;
}

// Tile L of (row tiles of BN padded rows) x n columns: within an expert the row tiles of a
// column are neighbours, so that they read its weights at the same time (160M, 1152 tokens: all
// columns of a row tile in a row 126 us, so 116; 1.3B, 500 tokens 901, 835).
struct RowTile {
  int e, p0, col;
  int l0, valid;  // first list entry, rows that are not padding
};
template <int BN>
__device__ __forceinline__ int row_tiles(const PadScan &g, int n, int &incl) {
  const int lane = threadIdx.x & 63;
  incl = (g.pc + BN - 1) / BN;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(incl, d, 64);
    if (lane >= d) incl += x;
  }
  return __builtin_amdgcn_readfirstlane(__shfl(incl, 63, 64)) * n;
}
template <int BN>
__device__ __forceinline__ RowTile row_tile(const PadScan &g, int incl, int n, int L) {
  const int nt = (g.pc + BN - 1) / BN;
  const uint64_t m = __ballot(incl * n > L);
  const int l = __ffsll((unsigned long long)m) - 1;
  const int nte = __builtin_amdgcn_readfirstlane(__shfl(nt, l, 64));
  const int x = __builtin_amdgcn_readfirstlane(L - (__shfl(incl, l, 64) - nte) * n), i = x % nte;
  RowTile r;
  r.e = __builtin_amdgcn_readfirstlane(l + 1);
  r.col = x / nte;
  r.p0 = __builtin_amdgcn_readfirstlane(__shfl(g.pad, l, 64) + i * BN);
  r.l0 = __builtin_amdgcn_readfirstlane(__shfl(g.list, l, 64) + i * BN);
  r.valid = __builtin_amdgcn_readfirstlane(min(BN, __shfl(g.c, l, 64) - i * BN));
  return r;
}

// ------------------------------------------------------------------ rows
// One wave per padded row: the normalised row (in fp64, rounded once, the
// forward's arithmetic and so its bits) and the row of dx, its gate, and where its
// assignment lies; zeros for the padding.
constexpr int ROW_BLOCKS = 4096;  // (of 8 a CU at once; a launch is limited to 2^32 threads, the rows are not)
template <typename T>
__global__ __launch_bounds__(256) void moe_grad_rows_kernel(
    const T *__restrict__ x, const T *__restrict__ dx, const T *__restrict__ g,
    const float *__restrict__ egate, const int32_t *__restrict__ cnt,
    const int32_t *__restrict__ rows, int E, int k, int d, float eps, T *__restrict__ n2,
    T *__restrict__ dy, float *__restrict__ gate, int32_t *__restrict__ row_of,
    int32_t *__restrict__ list_of) {
  const int lane = threadIdx.x & 63;
  const PadScan ps = pad_scan(cnt, E);
  for (int pos = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); pos < ps.total;
       pos += gridDim.x * 4) {
    const uint64_t m = __ballot(ps.pad + ps.pc > pos);
    const int l = __ffsll((unsigned long long)m) - 1;
    const int i = pos - __shfl(ps.pad, l, 64);
    T *no = n2 + int64_t(pos) * d, *yo = dy + int64_t(pos) * d;
    if (i >= __shfl(ps.c, l, 64)) {
      const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int c = lane * 8; c < d; c += 512) {
        store8(no + c, z);
        store8(yo + c, z);
      }
      if (lane == 0) gate[pos] = 0.f;
      continue;
    }
    const int entry = __shfl(ps.list, l, 64) + i;
    const int a = __builtin_amdgcn_readfirstlane(rows[entry]);
    const T *xr = x + int64_t(a / k) * d, *yr = dx + int64_t(a / k) * d;
    double ss = 0.0;
    for (int c = lane * 8; c < d; c += 512) {
      float w[8];
      load8(xr + c, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fma(double(w[j]), double(w[j]), ss);
    }
    ss = wave_sum(ss);
    const double r = 1.0 / sqrt(ss / double(d) + double(eps));
    for (int c = lane * 8; c < d; c += 512) {
      float w[8], gv[8], y[8];
      double o[8];
      load8(xr + c, w);
      load8(g + c, gv);
      load8(yr + c, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = (double(w[j]) * r) * double(gv[j]);
      store8(no + c, o);
      store8(yo + c, y);
    }
    if (lane == 0) {
      gate[pos] = egate[a];
      row_of[a] = pos;
      list_of[a] = entry;
    }
  }
}

// ------------------------------------------------------------------ bf16 tile
typedef short s16x4_t __attribute__((ext_vector_type(4)));

// Where a stage keeps the 32-byte column block b of K row k of a transposed
// operand of R columns: the 4 K rows that 16 lanes read at once, and those of the next
// lane group, lie in different banks.
template <int R>
__device__ __forceinline__ int tswz(int k, int b) {
  if constexpr (R == 32)
    return b ^ ((k >> 3) & 1);  // four K rows a bank span
  else if constexpr (R == 64)
    return b ^ (((k >> 1) & 1) | (((k >> 3) & 1) << 1));  // two K rows a bank span
  else
    return b ^ ((k & 3) | (((k >> 3) & 1) << 2));
}
// The same for 16-byte chunk c of row r of a K-contiguous operand (rows of 128 bytes).
template <bool PAIR>
__device__ __forceinline__ int rswz(int r, int c) {
  if constexpr (PAIR)
    return c ^ ((((r >> 3) & 3) << 1) | ((r >> 1) & 1));
  else
    return swz<8>(r, c);
}

// acc += A B^T over nk steps of 128 bytes of the sum (64 bf16 or 32 fp32), A of MR
// and B of NR rows, WM x WN waves (of which this is number `wave`; nk + 1 barriers of the
// block, for S 1 2 nk), S stages in LDS.  AT / BT: the operand lies as K rows of MR / NR columns.
// Sources are given as functions (row, 16-byte chunk of its K step) or,
// transposed, (K row of the step, 16-byte chunk of its columns) -> address at
// step 0, and step -> bytes from there.  SPLIT 2: a wave's rows are taken in
// halves from the two halves of A (the units' gates and ups).
// fp32: of 16 sum indices lane group g holds 4 g .. 4 g + 3, and MFMA i (16x16x4) takes
// component i of both operands.
template <typename T, int MR, int NR, bool AT, bool BT, int SPLIT, int WM, int WN, int S>
struct TileCore {
  static constexpr bool F = sizeof(T) == 4;
  static constexpr int KB = 128 / int(sizeof(T));  // sum indices of a step
  static constexpr int NW = WM * WN, MI = MR / WM / 16, NI = NR / WN / 16;
  static constexpr int ABYTES = MR * 128, STAGE = (MR + NR) * 128, IPW = STAGE / 1024 / NW;
  static_assert(STAGE % (1024 * NW) == 0, "whole transfers");
  using Frag = typename std::conditional<F, f32x4_t, bf16x8_t>::type;  // 16 rows x 32 (fp32: 16) indices

  static constexpr int fmask(int R) { return R >= 64 ? 3 : R / 16 - 1; }
  // Source chunk of 16-byte chunk c of K row k in a stage of a transposed operand of R columns.
  template <int R>
  __device__ static __forceinline__ int tchunk(int k, int c) {
    if constexpr (F)
      return c ^ (((k >> 2) & fmask(R)) << 2);  // the lane groups' K rows 4 g + i in different banks (R 32: halves)
    else
      return tswz<R>(k, c >> 1) * 2 + (c & 1);
  }

  template <int R, bool TR>
  __device__ static __forceinline__ Frag frag(const uint8_t *base, int row0, int ks, int lane) {
    const int n = lane & 15, g = lane >> 4;
    if constexpr (!TR) {
      const int r = row0 + n;
      return *(const Frag *)(base + r * 128 + (swz<8>(r, ks * 4 + g) << 4));
    } else if constexpr (F) {
      f32x4_t v;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = *(const float *)(base + (16 * ks + 4 * g + i) * (4 * R) +
                                (((row0 >> 4) ^ (g & fmask(R))) * 16 + n) * 4);
      return v;
    } else {
      typedef __attribute__((address_space(3))) s16x4_t *P;
      s16x4_t h[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int k = 32 * ks + 8 * g + 4 * x + (n >> 2);
        h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (P)(base + k * (2 * R) + tswz<R>(k, row0 >> 4) * 32 + (lane & 3) * 8));
      }
      typedef short s16x8_t __attribute__((ext_vector_type(8)));
      const s16x8_t v = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8_t, v);
    }
  }

  template <class FA, class FB, class SA, class SB>
  __device__ static __forceinline__ void run(uint8_t *smem, int wave, FA &&fa, FB &&fb, SA &&astep, SB &&bstep,
                                             int nk, f32x4_t (&acc)[MI][NI]) {
    const int lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    const uint8_t *src[IPW];
#pragma unroll
    for (int j = 0; j < IPW; ++j) {
      int p = (wave * IPW + j) * 64 + lane;  // the 16-byte piece of the stage
      const bool isa = (wave * IPW + j) * 1024 < ABYTES;
      if (isa) {
        if constexpr (AT) {
          constexpr int CR = MR * int(sizeof(T)) / 16;  // chunks a K row
          src[j] = fa(p / CR, tchunk<MR>(p / CR, p % CR));
        } else {
          src[j] = fa(p / 8, swz<8>(p / 8, p % 8));
        }
      } else {
        p -= ABYTES / 16;
        if constexpr (BT) {
          constexpr int CR = NR * int(sizeof(T)) / 16;
          src[j] = fb(p / CR, tchunk<NR>(p / CR, p % CR));
        } else {
          src[j] = fb(p / 8, swz<8>(p / 8, p % 8));
        }
      }
    }
    const uint32_t sbase = lds_addr(smem) + wave * IPW * 1024;
    auto issue = [&](int kt, int stage) {
      const int64_t ao = astep(kt), bo = bstep(kt);
#pragma unroll
      for (int j = 0; j < IPW; ++j) {
        const bool isa = (wave * IPW + j) * 1024 < ABYTES;
        dma16(src[j] + (isa ? ao : bo), sbase + stage * STAGE + j * 1024);
      }
    };
#pragma unroll
    for (int s0 = 0; s0 < S - 1; ++s0)
      if (s0 < nk) issue(s0, s0);
    for (int kt = 0; kt < nk; ++kt) {
      if constexpr (S == 1) {
        issue(kt, 0);
        wait_vm<0>();
        __syncthreads();
      } else {
        wait_stages<IPW, S>(min(S - 2, nk - 1 - kt));
        __syncthreads();  // every wave's part of stage kt is in; stage kt - 1 is free
        if (kt + S - 1 < nk) issue(kt + S - 1, (kt + S - 1) % S);
      }
      const uint8_t *As = smem + (kt % S) * STAGE, *Bs = As + ABYTES;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        Frag b[NI];
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) b[ni] = frag<NR, BT>(Bs, wn * (NR / WN) + ni * 16, ks, lane);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
          constexpr int H = MI / SPLIT;  // 16-row blocks of a wave in each part of A
          const int row0 = (mi / H) * (MR / SPLIT) + wm * (MR / SPLIT / WM) + (mi % H) * 16;
          const Frag a = frag<MR, AT>(As, row0, ks, lane);
          if constexpr (F) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int ni = 0; ni < NI; ++ni)
                acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[ni][i], acc[mi][ni], 0, 0, 0);
          } else {
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
              acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[ni], acc[mi][ni], 0, 0, 0);
          }
        }
      }
      if (S == 1 && kt + 1 < nk) __syncthreads();
    }
    __syncthreads();  // every wave is done with the stages
  }
};

// 4 consecutive results to memory in the tensor's type.
__device__ __forceinline__ void put4(bf16 *o, float x, float y, float z, float w) {
  *(uint2 *)o = make_uint2(pk_bf16(x, y), pk_bf16(z, w));
}
__device__ __forceinline__ void put4(float *o, float x, float y, float z, float w) {
  *(f32x4_t *)o = f32x4_t{x, y, z, w};
}

template <int MI, int NI>
__device__ __forceinline__ void zero_acc(f32x4_t (&acc)[MI][NI]) {
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
}

struct MoeGradArgs {
  const void *Wg, *Wu, *Wd;
  const void *n2, *dy;  // [rows][d]
  // dGU [rows][2 d_ff]: 64 dG, the same units' dU, the next 64 dG, ..; Hp [rows][d_ff]:
  // p s G U (NULL: not wanted)
  void *dGU, *Hp;
  const float *gate;    // [rows]
  float *Y, *gpart;     // [rows][d]; [rows][GP]
  void *dWg, *dWu, *dWd;
  const int32_t *cnt;
  int E, d, f, GP;
};

// Gradients of the hidden row's two factors and its gate's share, from fp32
// G, U, q: h = s G U unscaled.
struct Hidden {
  float dg, du, hp, gq;
};
template <bool FAST>
__device__ __forceinline__ Hidden hidden_grad(float G, float U, float q, float p) {
  const float s = FAST ? __builtin_amdgcn_rcpf(1.0f + __expf(-G)) : 1.0f / (1.0f + expf(-G));
  const float a = G * s, h = a * U, pq = p * q;
  Hidden r;
  r.du = pq * a;
  r.dg = pq * U * (s * (1.0f + (G - a)));
  r.hp = p * h;
  r.gq = q * h;
  return r;
}

// ------------------------------------------ few rows, and fp32: small tiles
// With few rows an expert the products read each weight about once and the time
// is that of the stream: narrow tiles over all CUs, stages in flight ahead of the one
// in use.  The fp32 products, bound by the fp32 MFMA rate, run on the same tiles,
// several blocks a CU (160M, 2000 tokens: 96 TFLOP/s of the 154 of a large product; MFMA 69 %
// busy, 79 while the CU has a block).

// [G; U; q] of HID_F units and 64 rows: four waves make G and U while four make q, over
// the same number of steps (and barriers), and hand it over in LDS.
// HID_F 32, with four stages, where the tiles then still are no more than the CUs: twice the
// CUs share the stream of the weights and, in fp32, the products.
// (160M, 1 token, 64 tiles: two stages 14.2 us, three 12.0, 128 tiles of 32 units 9.7; 256 x 512 in
// fp32, 128 tokens, 48 tiles: 19.2, 96 of 32 units 12.9; 410M, 333 tokens, 704 tiles, two
// blocks a CU with two stages 46 us, one with three 50.  Tiles of 128 rows, one block a CU: 1.0 to 1.2
// times the time at 30 to 400 rows an expert.)
constexpr int HID_R = 64;
template <typename T, int HID_F, int HID_S>
__global__ __launch_bounds__(512) void moe_grad_hidden_kernel(MoeGradArgs a, int nf) {
  constexpr int WM = HID_F / 32, WN = 4 / WM;  // waves of 32 units
  using C1 = TileCore<T, 2 * HID_F, HID_R, false, false, 2, WM, WN, HID_S>;
  using C2 = TileCore<T, HID_F, HID_R, true, false, 1, WM, WN, HID_S>;
  constexpr int MI = C2::MI, NI = C2::NI, ES = sizeof(T);
  __shared__ __align__(1024) uint8_t smem[HID_S * (C1::STAGE + C2::STAGE)];
  const PadScan ps = pad_scan(a.cnt, a.E);
  int incl;
  const int total = row_tiles<HID_R>(ps, nf, incl);
  if (int(blockIdx.x) >= total) return;
  const RowTile t = row_tile<HID_R>(ps, incl, nf, xcd_tile(blockIdx.x, total));
  const int f0 = t.col * HID_F;
  const int d = a.d, f = a.f, steps = d / C1::KB;
  const int lane = threadIdx.x & 63, w8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = w8 & 3, wm = wave / WN, wn = wave % WN;
  auto along = [](int kt) { return int64_t(kt) * 128; };
  // (padding: one line, read again, instead of rows of zeros; 1.3B, 100 tokens 746 us, 729)
  auto row = [&](int r) { return r < t.valid ? r : 0; };
  f32x4_t(*qs)[64] = (f32x4_t(*)[64])(smem + HID_S * C1::STAGE) + wave * MI * NI;  // [block][lane]
  if (w8 >= 4) {
    const T *Wd = (const T *)a.Wd + int64_t(t.e - 1) * d * f + f0, *dy = (const T *)a.dy + int64_t(t.p0) * d;
    f32x4_t q[MI][NI];
    zero_acc(q);
    C2::run(
        smem + HID_S * C1::STAGE, wave, [&](int k, int c) { return (const uint8_t *)(Wd + int64_t(k) * f) + c * 16; },
        [&](int r, int c) { return (const uint8_t *)(dy + int64_t(row(r)) * d) + c * 16; },
        [&](int kt) { return int64_t(kt) * (C2::KB * ES) * f; }, along, steps, q);
#pragma unroll
    for (int i = 0; i < MI * NI; ++i) qs[i][lane] = q[i / NI][i % NI];
    __syncthreads();
    return;
  }
  const uint8_t *Wg = (const uint8_t *)((const T *)a.Wg + (int64_t(t.e - 1) * f + f0) * d);
  const int64_t up = (const uint8_t *)a.Wu - (const uint8_t *)a.Wg;
  const T *n2 = (const T *)a.n2 + int64_t(t.p0) * d;
  f32x4_t gu[2 * MI][NI];
  zero_acc(gu);
  C1::run(
      smem, wave,
      [&](int r, int c) { return Wg + (r / HID_F) * up + int64_t(r % HID_F) * ES * d + c * 16; },
      [&](int r, int c) { return (const uint8_t *)(n2 + int64_t(row(r)) * d) + c * 16; }, along, along, steps, gu);
  __syncthreads();  // q is there
#pragma unroll
  for (int ni = 0; ni < NI; ++ni) {
    const int r = wn * (HID_R / WN) + ni * 16 + (lane & 15);
    const int64_t pos = t.p0 + r;
    const bool live = r < t.valid;  // the padding's are zeros
    const float p = a.gate[pos];
    float gs = 0.f;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int u = f0 + wm * 32 + mi * 16 + 4 * (lane >> 4);
      const f32x4_t q = qs[mi * NI + ni][lane];
      Hidden h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = hidden_grad<ES == 2>(live ? gu[mi][ni][i] : 0.f, live ? gu[MI + mi][ni][i] : 0.f,
                                    live ? q[i] : 0.f, p);
        gs += h[i].gq;
      }
      T *o = (T *)a.dGU + pos * (2 * f) + (u & ~63) + u;
      put4(o, h[0].dg, h[1].dg, h[2].dg, h[3].dg);
      put4(o + 64, h[0].du, h[1].du, h[2].du, h[3].du);
      if (a.Hp) put4((T *)a.Hp + pos * f + u, h[0].hp, h[1].hp, h[2].hp, h[3].hp);
    }
    gs += __shfl_xor(gs, 16, 64);
    gs += __shfl_xor(gs, 32, 64);
    if (lane < 16) a.gpart[pos * a.GP + f0 / 32 + wm] = gs;
  }
}

// dn of 64 columns and 64 rows over one of `splits` parts of the sum, to its plane
// of Y (list order).
constexpr int INP_M = 64, INP_R = 64;
template <typename T>
using InputCore = TileCore<T, INP_M, INP_R, true, false, 1, 2, 2, 2>;
template <typename T>
__device__ __forceinline__ void input_tile(const MoeGradArgs &a, uint8_t *smem, int block, int nd, int splits,
                                           int64_t plane) {
  using C = InputCore<T>;
  constexpr int ES = sizeof(T), SPB = 64 / C::KB;  // steps of 64 gates (ups)
  const PadScan ps = pad_scan(a.cnt, a.E);
  int incl;
  const int total = row_tiles<INP_R>(ps, nd * splits, incl);
  if (block >= total) return;
  const RowTile t = row_tile<INP_R>(ps, incl, nd * splits, xcd_tile(block, total));
  const int sp = t.col % splits;
  const int m0 = (t.col / splits) * INP_M, d = a.d, f = a.f, blocks = f / 64;
  const int h0 = int(int64_t(blocks) * sp / splits), h1 = int(int64_t(blocks) * (sp + 1) / splits);
  const T *Wg = (const T *)a.Wg + (int64_t(t.e - 1) * f + h0 * 64) * d + m0;
  const T *g = (const T *)a.dGU + int64_t(t.p0) * (2 * f) + h0 * 128;
  const int64_t up = (const uint8_t *)a.Wu - (const uint8_t *)a.Wg;
  f32x4_t acc[C::MI][C::NI];
  zero_acc(acc);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / 2, wn = wave % 2;
  C::run(
      smem, wave, [&](int k, int c) { return (const uint8_t *)(Wg + int64_t(k) * d) + c * 16; },
      [&](int r, int c) { return (const uint8_t *)(g + int64_t(r) * (2 * f)) + c * 16; },
      [&](int kt) {  // 64 rows of Wg, the same of Wu, the next of Wg ..
        const int x = kt / SPB;
        return int64_t((x >> 1) * 64 + (kt % SPB) * C::KB) * ES * d + (x & 1) * up;
      },
      [](int kt) { return int64_t(kt) * 128; }, 2 * SPB * (h1 - h0), acc);
#pragma unroll
  for (int ni = 0; ni < C::NI; ++ni) {
    const int r = wn * (INP_R / 2) + ni * 16 + (lane & 15);
    if (r >= t.valid) continue;
    float *y = a.Y + sp * plane + int64_t(t.l0 + r) * d + m0 + wm * (INP_M / 2) + 4 * (lane >> 4);
#pragma unroll
    for (int mi = 0; mi < C::MI; ++mi) *(f32x4_t *)(y + mi * 16) = acc[mi][ni];
  }
}

// 128 x 128 of an expert's weight gradients (see WeightBig).  bf16: written in rows of
// 256 bytes through LDS (with few rows it is the time of the writes; one stage and four
// blocks a CU: 160M, 1 token 17.4 us, three blocks 20.4; 410M, 333 tokens 39.5, 45.0).  Two stages
// and two blocks a CU instead, the whole pass: 160M, 1 token 43 us, 50; 2000 tokens 169, 186, in fp32
// 867, 879; only layers of few tiles with many rows gain (256 x 512, 4 experts, 8000 tokens 81, 68).
constexpr int WGT_T = 128;
template <typename T>
using WeightCore = TileCore<T, WGT_T, WGT_T, true, true, 1, 2, 2, 1>;
template <typename T>
__device__ __forceinline__ void weight_tile(const MoeGradArgs &a, uint8_t *smem, int block, int tiles) {
  using C = WeightCore<T>;
  constexpr int ES = sizeof(T), EC = 16 / ES;  // elements of a chunk
  const int d = a.d, f = a.f;
  const int md = (d + WGT_T - 1) / WGT_T, mf = (f + WGT_T - 1) / WGT_T;
  const int t1 = md * (2 * f / WGT_T), t2 = mf * md;  // (2 f is a multiple of 128)
  int L = xcd_tile(block, tiles);
  const int e = L / (t1 + t2) + 1;
  L -= (e - 1) * (t1 + t2);
  const PadScan ps = pad_scan(a.cnt, a.E);
  const int p0 = __builtin_amdgcn_readfirstlane(__shfl(ps.pad, e - 1, 64));
  const int rows = __builtin_amdgcn_readfirstlane(__shfl(ps.pc, e - 1, 64));
  const bool down = L >= t1;  // dWd[d][f] = dy^T Hp; else [dWg; dWu] = dGU^T n2
  if (down) L -= t1;
  const int mt = down ? mf : md, M = down ? f : d, N = down ? d : 2 * f;
  const int m0 = (L % mt) * WGT_T, n0 = (L / mt) * WGT_T;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / 2, wn = wave % 2;
  // row n of the tile's matrix: of dWd, or 64 units of dWg, the same of dWu, ..
  auto out_row = [&](int n) {
    T *o = (T *)(down ? a.dWd : (n & 64) ? a.dWu : a.dWg) + int64_t(e - 1) * d * f;
    return o + int64_t(down ? n : (n >> 7) * 64 + (n & 63)) * M + m0;
  };
  if (rows > 0) {
    const T *A = (const T *)(down ? a.Hp : a.n2) + int64_t(p0) * M + m0;
    const T *B = (const T *)(down ? a.dy : a.dGU) + int64_t(p0) * N + n0;
    f32x4_t acc[C::MI][C::NI];
    zero_acc(acc);
    C::run(
        smem, wave, [&](int k, int c) { return (const uint8_t *)(A + int64_t(k) * M) + (m0 + c * EC < M ? c * 16 : 0); },
        [&](int k, int c) { return (const uint8_t *)(B + int64_t(k) * N) + (n0 + c * EC < N ? c * 16 : 0); },
        [&](int kt) { return int64_t(kt) * 128 * M; }, [&](int kt) { return int64_t(kt) * 128 * N; }, rows / C::KB,
        acc);
#pragma unroll
    for (int ni = 0; ni < C::NI; ++ni)
#pragma unroll
      for (int mi = 0; mi < C::MI; ++mi) {
        const int n = wn * 64 + ni * 16 + (lane & 15), m = wm * 64 + mi * 16 + 4 * (lane >> 4);
        const f32x4_t v = acc[mi][ni];
        if constexpr (ES == 4) {
          if (n0 + n < N && m0 + m < M) put4(out_row(n0 + n) + m, v[0], v[1], v[2], v[3]);
        } else {
          // row n of 256 bytes, its 16-byte chunks turned by the row
          put4((T *)(smem + n * 256 + (((m >> 3) ^ (n & 15)) << 4) + (m & 4) * 2), v[0], v[1], v[2], v[3]);
        }
      }
    if constexpr (ES == 4) return;
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < WGT_T * (WGT_T / EC) / 256; ++x) {
    constexpr int CR = WGT_T / EC;  // chunks a row
    const int r = x * (256 / CR) + tid / CR, c = tid % CR;
    if (n0 + r >= N || m0 + c * EC >= M) continue;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (ES == 2 && rows > 0) v = *(const uint4 *)(smem + r * 256 + ((c ^ (r & 15)) << 4));
    *(uint4 *)(out_row(n0 + r) + c * EC) = v;
  }
}

// dn alone (frozen experts), or dn's tiles (the first nin blocks) beside the weight
// gradients', which do not wait for each other.
template <typename T>
__global__ __launch_bounds__(256) void moe_grad_input_kernel(MoeGradArgs a, int nd, int splits, int64_t plane) {
  __shared__ __align__(1024) uint8_t smem[2 * InputCore<T>::STAGE];
  input_tile<T>(a, smem, blockIdx.x, nd, splits, plane);
}
template <typename T>
__global__ __launch_bounds__(256, 4) void moe_grad_input_weight_kernel(
    MoeGradArgs a, int nin, int nd, int splits, int64_t plane) {
  constexpr int BI = 2 * InputCore<T>::STAGE, BW = WeightCore<T>::STAGE;
  __shared__ __align__(1024) uint8_t smem[BI > BW ? BI : BW];
  if (int(blockIdx.x) < nin)
    input_tile<T>(a, smem, blockIdx.x, nd, splits, plane);
  else
    weight_tile<T>(a, smem, int(blockIdx.x) - nin, int(gridDim.x) - nin);
}

// ------------------------------------------------------- four-wave products
// One block a CU, one wave a SIMD, 256 x 256 tiles walked by a resident block: 128 x 128 to a
// wave, so that a fragment read from LDS feeds eight MFMAs.  1.3B, 16384 tokens, means of ten calls: q
// 733 us, gates and ups 1414, dn and the weights 3080 (970, 1005 and 1155 TFLOP/s; the fastest of the
// ten 697, 1362 and 2890; MFMA 53, 53 and 64 % busy at the 1.8 GHz that the chip's power leaves).  The loops alone run at 1260-1450, a large library product's
// rate; the rest is what an epilogue reads, computes and writes, 0.2 to 0.3 MB a tile.  Stages of 64
// sum indices, two of them in LDS; the fragments of the next 32 are read
// while the MFMAs of the present 32 issue.  The transfers run on over the
// tiles' ends: the producer is two stages ahead in the block's list of (tile, step), whatever
// the tiles' own numbers of steps.
struct BigTile {
  int e, p0, rows, m0, n0, nk, down;
};
// Column tiles of a product over row tiles (ny), or the weight product's: column tiles of d
// and d_ff, tiles of its two problems.
struct BigShape {
  int ny, md, mf, t1, t2;
};

// One operand of a stage: R rows of 64 sum indices (K-contiguous), or 64 rows of R
// columns (TR).  The 1 KB transfers are dealt to the four waves in turn; the
// jj-th of a wave covers K rows (rows) RPJ jj on.
template <int R, bool TR, bool PAIR>
struct Operand {
  static constexpr int BYTES = R * 128, XF = BYTES / 4096;
  static constexpr int RPJ = TR ? 2048 / R : 32;
  static constexpr int PAR = TR && R == 256 ? 2 : 1;
  // the lane's source offset; columns from `valid` on (TR) read the first ones
  // instead (their products are never stored)
  __device__ static __forceinline__ uint32_t offset(int wave, int lane, int par, uint32_t ld, int valid) {
    if constexpr (!TR) {
      const int r = 8 * wave + (lane >> 3);
      return uint32_t(r) * ld + rswz<PAIR>(r, lane & 7) * 16;
    } else {
      constexpr int LPR = R / 8;  // lanes a K row
      const int k = (64 / LPR) * wave + lane / LPR, c = lane % LPR;
      int cc = tswz<R>(k + RPJ * par, c >> 1) * 2 + (c & 1);
      cc = cc * 8 < valid ? cc : 0;
      return uint32_t(k) * ld + cc * 16;
    }
  }
};

// A wave-uniform pointer that the compiler would otherwise keep in vector registers.
__device__ __forceinline__ const uint8_t *uniform(const void *p) {
  const uint64_t u = uint64_t(uintptr_t(p));
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(u)), hi = __builtin_amdgcn_readfirstlane(uint32_t(u >> 32));
  return (const uint8_t *)uintptr_t(lo | (uint64_t(hi) << 32));
}

// The producer's view of an operand: the base of its present stage (scalar) and the
// lane's byte offset of each of the wave's transfers from it.
template <int R, bool TR, bool PAIR = false>
struct Src {
  using O = Operand<R, TR, PAIR>;
  const uint8_t *cur;
  int64_t step;  // bytes from one stage to the next
  uint32_t off[O::XF];
  // rows: rows to read (K-contiguous; a multiple of 64 or all of them): the others read the first;
  // cols: columns to read (TR)
  __device__ __forceinline__ void init(const void *base, int64_t ld_elems, int64_t step_, int rows, int cols) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    cur = uniform(base);
    step = step_;
    const uint32_t ld = uint32_t(ld_elems * 2);
    uint32_t o[O::PAR];
#pragma unroll
    for (int p = 0; p < O::PAR; ++p) o[p] = O::offset(wave, lane, p, ld, cols);
#pragma unroll
    for (int j = 0; j < O::XF; ++j) {
      const int row = O::RPJ * j;
      off[j] = o[O::PAR == 2 ? j & 1 : 0] + (TR || row < rows ? uint32_t(row) * ld : 0u);
    }
  }
};

// One transfer (dma16_s) to LDS address lds + OFF beside one MFMA, which also is the
// wait state between the write of m0 and its use: two more instructions in the
// shadow of the product, where an address of its own would cost five.
template <bool FIRST, int OFF>
__device__ __forceinline__ void mfma_dma(f32x4_t &acc, const bf16x8_t &a, const bf16x8_t &b, const void *base,
                                         uint32_t voff, uint32_t lds) {
  if constexpr (FIRST)
    asm volatile(
        "s_add_u32 m0, %4, %6\n\t"
        "v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0\n\t"
        "global_load_lds_dwordx4 %3, %5"
        : "=a"(acc)
        : "v"(a), "v"(b), "v"(voff), "s"(lds), "s"(base), "i"(OFF)
        : "memory", "m0", "scc");
  else
    asm volatile(
        "s_add_u32 m0, %4, %6\n\t"
        "v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0\n\t"
        "global_load_lds_dwordx4 %3, %5"
        : "+a"(acc)
        : "v"(a), "v"(b), "v"(voff), "s"(lds), "s"(base), "i"(OFF)
        : "memory", "m0", "scc");
}

// Fragment addresses (LDS) of an operand in the present stage: 16 rows of block i
// from row0 on.  What differs by block or slice is an immediate offset, and the
// switch to the other stage (flip) one addition an address and step.
// PAIR (K-contiguous): row 4 q + t of blocks 2 j and 2 j + 1 is operand row 32 j + 8 q + t and
// 32 j + 8 q + 4 + t, so that a lane's results of the two blocks are 8 consecutive ones: one
// 16-byte store in bf16, four lanes a 64-byte run.  (The transposing load would read 8
// bytes of every 16 then, and half the banks: see pair_rows.)
template <int R, bool TR, bool PAIR, int NI>
struct Frags {
  static_assert(!(TR && PAIR), "K-contiguous operands");
  static constexpr int NB = TR ? NI : 2;
  uint32_t b[NB];
  __device__ __forceinline__ void init(uint32_t base, int row0, int lane) {
    const int n = lane & 15;
    if constexpr (!TR) {
      const int r = row0 + (PAIR ? (n >> 2) * 8 + (n & 3) : n);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) b[ks] = base + r * 128 + (rswz<PAIR>(r, ks * 4 + (lane >> 4)) << 4);
    } else {
      const int k = 8 * (lane >> 4) + (n >> 2), q = lane & 3;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int col = row0 + i * 16 + q * 4;
        b[i] = base + k * (2 * R) + tswz<R>(k, col >> 4) * 32 + (col & 15) * 2;
      }
    }
  }
  __device__ __forceinline__ void flip(int delta) {
#pragma unroll
    for (int i = 0; i < NB; ++i) b[i] += delta;
  }
  __device__ __forceinline__ bf16x8_t read(int ks, int i) const {
    if constexpr (!TR) {
      typedef const __attribute__((address_space(3))) bf16x8_t *P;
      return *(P)(b[ks] + (PAIR ? (i >> 1) * 4096 + (i & 1) * 512 : i * 2048));
    } else {
      typedef __attribute__((address_space(3))) s16x4_t *P;
      const uint32_t a = b[i] + ks * (64 * R);
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)a);
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(a + 8 * R));
      return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Row tiles of BN rows of every expert (lane e - 1), their inclusive sums.
struct TileScan {
  PadScan ps;
  int nt, incl, total;
};
template <int BN>
__device__ __forceinline__ TileScan tile_scan(const int32_t *cnt, int E) {
  TileScan g;
  g.ps = pad_scan(cnt, E);
  g.nt = (g.ps.pc + BN - 1) / BN;
  int x = g.nt;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  g.incl = x;
  g.total = __builtin_amdgcn_readfirstlane(__shfl(x, 63, 64));
  return g;
}
// Tile t of (row tiles x ny columns), in bands of BR x BC tiles within each expert: the 32
// blocks of an XCD then read BR + BC operand slices.  (1.3B, 16384 tokens, 16 x 2 / 4 x 8,
// us: weights 1824 / 1794, dn 1126 / 1116; 160M dn 227 / 206, gates 284 / 278; q, whose tiles are
// shortest, 723 / 732 and 684 with 6 x 5.)
template <int BN, int BR, int BC>
__device__ __forceinline__ BigTile row_col_tile(const TileScan &g, int t, int ny, int &col) {
  const uint64_t m = __ballot(g.incl * ny > t);
  const int l = __ffsll((unsigned long long)m) - 1;
  const int nt = __shfl(g.nt, l, 64), first = __shfl(g.incl, l, 64) - nt;
  int i;
  band_order<BR, BC>(t - first * ny, nt, ny, i, col);
  BigTile r;
  r.e = __builtin_amdgcn_readfirstlane(l + 1);
  r.p0 = __builtin_amdgcn_readfirstlane(__shfl(g.ps.pad, l, 64) + i * BN);
  r.rows = __builtin_amdgcn_readfirstlane(min(BN, __shfl(g.ps.pc, l, 64) - i * BN));
  col = __builtin_amdgcn_readfirstlane(col);
  r.down = 0;
  return r;
}

// An accumulator's values, read where they are used: left to itself the compiler copies
// all of them to vector registers at once, and spills.
__device__ __forceinline__ f32x4_t acc_get(const f32x4_t &a) {
  f32x4_t v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[0]) : "a"(a[0]));
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[1]) : "a"(a[1]));
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[2]) : "a"(a[2]));
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[3]) : "a"(a[3]));
  return v;
}

// Shared by the products over row tiles of 256: out [rows][..] of A's 256 rows (columns of a
// weight) against the rows of a tile.
struct RowsBase {
  static constexpr bool EMPTY = false;  // a tile may have no steps
  static constexpr int BN = 256, MI = 8, NI = 8, NA = 8, NB = 8;
  static constexpr int STAGE = 2 * 32768, IPW = 16, NM = 64;
  const MoeGradArgs &a;  // the kernel's own argument, which is not written
  const int ny;
  __device__ __forceinline__ RowsBase(const MoeGradArgs &a_, const BigShape &s) : a(a_), ny(s.ny) {}
  __device__ __forceinline__ TileScan scan() const { return tile_scan<BN>(a.cnt, a.E); }
  __device__ __forceinline__ int total(const TileScan &g) const { return g.total * ny; }
  static constexpr int lds_off(int j) { return j * 4096; }
};

// fp32 out = W^T rows, 256 columns of W (whose rows are the sum index) and 256 rows.
// TWO: dn = Wg^T dG + Wu^T dU; else q = Wd^T dx.
template <bool TWO>
struct RowsBig : RowsBase {
  using RowsBase::RowsBase;
  static constexpr int BR = TWO ? 4 : 6, BC = TWO ? 8 : 5;
  Src<256, true> sw;
  Src<256, false> sr;
  const uint8_t *other;  // the next stage of the matrix whose turn it is not
  Frags<256, true, false, 8> fa_;
  Frags<256, false, false, 8> fb_;
  __device__ __forceinline__ BigTile tile(const TileScan &g, int l, int total) const {
    int by;
    BigTile t = row_col_tile<BN, BR, BC>(g, xcd_tile(l, total), ny, by);
    t.m0 = by * 256;
    t.n0 = 0;
    t.nk = TWO ? a.f / 32 : a.d / 64;
    return t;
  }
  __device__ __forceinline__ void source(const BigTile &t) {
    const int64_t d = a.d, f = a.f, w = int64_t(t.e - 1) * f * d + t.m0;
    if constexpr (TWO) {
      sw.init((const bf16 *)a.Wg + w, d, 128 * d, 0, a.d - t.m0);
      other = uniform((const bf16 *)a.Wu + w);
      sr.init((const bf16 *)a.dGU + int64_t(t.p0) * (2 * f), 2 * f, 128, t.rows, 0);
    } else {
      sw.init((const bf16 *)a.Wd + w, f, 128 * f, 0, a.f - t.m0);
      sr.init((const bf16 *)a.dy + int64_t(t.p0) * d, d, 128, t.rows, 0);
    }
  }
  __device__ __forceinline__ void next(int) {
    if constexpr (TWO) {  // 64 gates, then the same 64 ups
      const uint8_t *n = sw.cur + sw.step;
      sw.cur = other;
      other = n;
    } else {
      sw.cur += sw.step;
    }
    sr.cur += sr.step;
  }
  __device__ __forceinline__ const uint8_t *base(int j) const { return j < 8 ? sw.cur : sr.cur; }
  __device__ __forceinline__ uint32_t off(int j) const { return j < 8 ? sw.off[j & 7] : sr.off[j & 7]; }
  __device__ __forceinline__ void frags(uint32_t smem, int wm, int wn, int lane) {
    fa_.init(smem, wm * 128, lane);
    fb_.init(smem + 32768, wn * 128, lane);
  }
  __device__ __forceinline__ void flip(int delta) {
    fa_.flip(delta);
    fb_.flip(delta);
  }
  // piece q of slice ks, in the order of their first use: A0, the rows, A1 ..
  __device__ __forceinline__ void read(int q, int ks, bf16x8_t (&fa)[NA], bf16x8_t (&fb)[NB]) const {
    if (q == 0) fa[0] = fa_.read(ks, 0);
    else if (q <= NB) fb[q - 1] = fb_.read(ks, q - 1);
    else fa[q - NB] = fa_.read(ks, q - NB);
  }
  __device__ __forceinline__ void store(const BigTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn,
                                        int lane) const {
    const int M = TWO ? a.d : a.f;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      const int r = wn * 128 + ni * 16 + (lane & 15);
      if (r >= t.rows) continue;
      float *y = (TWO ? a.Y : (float *)a.dGU) + int64_t(t.p0 + r) * M;
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int m = t.m0 + wm * 128 + mi * 16 + 4 * (lane >> 4);
        if (m < M) *(f32x4_t *)(y + m) = acc[mi][ni];
      }
    }
  }
};

// G and U of 128 units and 256 rows, and with q (in fp32, where dG and dU go) the
// hidden gradients: A blocks 0..3 are a wave's gates, 4..7 its ups.
struct GateUpBig : RowsBase {
  using RowsBase::RowsBase;
  static constexpr int BR = 4, BC = 8;
  Src<128, false, true> sg, su;
  Src<256, false> sr;
  Frags<128, false, true, 4> fg, fu;
  Frags<256, false, false, 8> fb_;
  __device__ __forceinline__ BigTile tile(const TileScan &g, int l, int total) const {
    int by;
    BigTile t = row_col_tile<BN, BR, BC>(g, xcd_tile(l, total), ny, by);
    t.m0 = by * 128;
    t.n0 = 0;
    t.nk = a.d / 64;
    return t;
  }
  __device__ __forceinline__ void source(const BigTile &t) {
    const int64_t d = a.d, w = (int64_t(t.e - 1) * a.f + t.m0) * d;
    const int uv = min(128, a.f - t.m0);
    sg.init((const bf16 *)a.Wg + w, d, 128, uv, 0);
    su.init((const bf16 *)a.Wu + w, d, 128, uv, 0);
    sr.init((const bf16 *)a.n2 + int64_t(t.p0) * d, d, 128, t.rows, 0);
  }
  __device__ __forceinline__ void next(int) {
    sg.cur += sg.step;
    su.cur += su.step;
    sr.cur += sr.step;
  }
  __device__ __forceinline__ const uint8_t *base(int j) const { return j < 4 ? sg.cur : j < 8 ? su.cur : sr.cur; }
  __device__ __forceinline__ uint32_t off(int j) const {
    return j < 4 ? sg.off[j & 3] : j < 8 ? su.off[j & 3] : sr.off[j & 7];
  }
  __device__ __forceinline__ void frags(uint32_t smem, int wm, int wn, int lane) {
    fg.init(smem, wm * 64, lane);
    fu.init(smem + 16384, wm * 64, lane);
    fb_.init(smem + 32768, wn * 128, lane);
  }
  __device__ __forceinline__ void flip(int delta) {
    fg.flip(delta);
    fu.flip(delta);
    fb_.flip(delta);
  }
  __device__ __forceinline__ void read(int q, int ks, bf16x8_t (&fa)[NA], bf16x8_t (&fb)[NB]) const {
    if (q == 0) fa[0] = fg.read(ks, 0);
    else if (q <= NB) fb[q - 1] = fb_.read(ks, q - 1);
    else if (q - NB < 4) fa[q - NB] = fg.read(ks, q - NB);
    else fa[q - NB] = fu.read(ks, q - NB - 4);
  }
  __device__ __forceinline__ void store(const BigTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn,
                                        int lane) const {
    const int u0 = t.m0 + wm * 64, f = a.f;
    if (u0 >= f) return;
    // The lane's 8 units of each half of the wave's 64: their q (256 bytes a row) are read before
    // dG and dU take their place; nothing but the row's other three lanes touches
    // those bytes, in the same instructions.  The q of NQ row blocks are in flight, asked for before the
    // stores of the block NQ before them: loads and stores are waited for in their order.
    const int u = 8 * (lane >> 4);
    constexpr int NQ = 4;
    f32x4_t q[NQ][2][2];
    float p[NQ];
    auto load = [&](int ni) __attribute__((always_inline)) {
      const int r = wn * 128 + ni * 16 + (lane & 15);
      const int64_t pos = t.p0 + (r < t.rows ? r : 0);  // (the first row's are read, and not used)
      const float *qr = (const float *)a.dGU + pos * f + u0 + u;
      p[ni % NQ] = a.gate[pos];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) q[ni % NQ][j][h] = *(const f32x4_t *)(qr + 32 * j + 4 * h);
    };
#pragma unroll
    for (int ni = 0; ni < NQ; ++ni) load(ni);
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      const int r = wn * 128 + ni * 16 + (lane & 15), n = ni % NQ;
      const int64_t pos = t.p0 + r;
      const bool in = r < t.rows;
      float gs = 0.f;
      uint4 wg[2], wu[2], wh[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        Hidden h[8];
        const f32x4_t G[2] = {acc_get(acc[2 * j][ni]), acc_get(acc[2 * j + 1][ni])};
        const f32x4_t U[2] = {acc_get(acc[4 + 2 * j][ni]), acc_get(acc[5 + 2 * j][ni])};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[i] = hidden_grad<true>(G[i >> 2][i & 3], U[i >> 2][i & 3], q[n][j][i >> 2][i & 3], p[n]);
          gs += h[i].gq;
        }
        wg[j] = make_uint4(pk_bf16(h[0].dg, h[1].dg), pk_bf16(h[2].dg, h[3].dg),
                           pk_bf16(h[4].dg, h[5].dg), pk_bf16(h[6].dg, h[7].dg));
        wu[j] = make_uint4(pk_bf16(h[0].du, h[1].du), pk_bf16(h[2].du, h[3].du),
                           pk_bf16(h[4].du, h[5].du), pk_bf16(h[6].du, h[7].du));
        wh[j] = make_uint4(pk_bf16(h[0].hp, h[1].hp), pk_bf16(h[2].hp, h[3].hp),
                           pk_bf16(h[4].hp, h[5].hp), pk_bf16(h[6].hp, h[7].hp));
      }
      __builtin_amdgcn_sched_barrier(0);
      if (ni + NQ < NI) load(ni + NQ);
      __builtin_amdgcn_sched_barrier(0);
      gs += __shfl_xor(gs, 16, 64);
      gs += __shfl_xor(gs, 32, 64);
      if (in) {
        bf16 *o = (bf16 *)a.dGU + pos * (2 * f) + 2 * u0 + u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          *(uint4 *)(o + 32 * j) = wg[j];
          *(uint4 *)(o + 64 + 32 * j) = wu[j];
          if (a.Hp) *(uint4 *)((bf16 *)a.Hp + pos * f + u0 + 32 * j + u) = wh[j];
        }
        if (lane < 16) a.gpart[pos * a.GP + u0 / 64] = gs;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Rows 4 g .. 4 g + 3 (g = lane / 16) of two 16-row blocks a and b, packed, to 8
// consecutive rows a lane: lane groups 0 and 2 get rows 0 .. 7 and 8 .. 15 of a, 1 and 3
// those of b (the odd groups' words of a change places with the even groups' of b).
__device__ __forceinline__ uint4 pair_rows(uint2 a, uint2 b) {
  const auto x = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}

// 256 x 256 of an expert's weight gradients: [dWg; dWu] (columns d of n2
// against units of [dG dU]) or, down, dWd (units of p s G U against columns d of
// dy); the sum runs over the expert's rows.  The tiles of an expert are dealt to all
// XCDs, so that experts with many rows load them alike.
struct WeightBig {
  static constexpr bool EMPTY = true;
  static constexpr int MI = 8, NI = 8, NA = 8, NB = 8;
  static constexpr int STAGE = 2 * 32768, IPW = 16, NM = 64;
  const MoeGradArgs &a;
  const int md, mf, t1, t2;
  __device__ __forceinline__ WeightBig(const MoeGradArgs &a_, const BigShape &s)
      : a(a_), md(s.md), mf(s.mf), t1(s.t1), t2(s.t2) {}
  Src<256, true> sm, sn;
  Frags<256, true, false, 8> fa_, fb_;
  __device__ __forceinline__ TileScan scan() const {
    TileScan g;
    g.ps = pad_scan(a.cnt, a.E);
    return g;
  }
  // row n of the tile's matrix: a unit's row of dWg or dWu, or a column's of dWd
  __device__ __forceinline__ bf16 *out_row(const BigTile &t, int n) const {
    const int64_t e = int64_t(t.e - 1) * a.d * a.f;
    if (t.down) return (bf16 *)a.dWd + e + int64_t(n) * a.f;
    const int u = (n >> 7) * 64 + (n & 63);  // 64 gates, then the same 64 ups
    return (bf16 *)((n & 64) ? a.dWu : a.dWg) + e + int64_t(u) * a.d;
  }
  __device__ __forceinline__ void store_zero(const BigTile &t) const {
    const int M = t.down ? a.f : a.d, N = t.down ? a.d : 2 * a.f;
    const int m = t.m0 + (threadIdx.x & 31) * 8;
    for (int r = threadIdx.x >> 5; r < 256; r += 8)
      if (t.n0 + r < N && m < M) *(uint4 *)(out_row(t, t.n0 + r) + m) = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ int total(const TileScan &) const { return a.E * (t1 + t2); }
  __device__ __forceinline__ BigTile tile(const TileScan &g, int l, int) const {
    BigTile t;
    const int e = l / (t1 + t2);
    int x = xcd_tile(l - e * (t1 + t2), t1 + t2), i, j;
    t.down = x >= t1;
    if (t.down) {
      x -= t1;
      band_order<4, 8>(x, md, mf, j, i);
    } else {
      band_order<4, 8>(x, t1 / md, md, j, i);
    }
    t.e = e + 1;
    t.p0 = __builtin_amdgcn_readfirstlane(__shfl(g.ps.pad, e, 64));
    t.rows = __builtin_amdgcn_readfirstlane(__shfl(g.ps.pc, e, 64));
    t.nk = t.rows / 64;
    t.m0 = i * 256;
    t.n0 = j * 256;
    return t;
  }
  __device__ __forceinline__ void source(const BigTile &t) {
    const int64_t M = t.down ? a.f : a.d, N = t.down ? a.d : 2 * a.f;
    sm.init((const bf16 *)(t.down ? a.Hp : a.n2) + t.p0 * M + t.m0, M, 128 * M, 0, int(M) - t.m0);
    sn.init((const bf16 *)(t.down ? a.dy : a.dGU) + t.p0 * N + t.n0, N, 128 * N, 0, int(N) - t.n0);
  }
  __device__ __forceinline__ void next(int) {
    sm.cur += sm.step;
    sn.cur += sn.step;
  }
  static constexpr int lds_off(int j) { return j * 4096; }
  __device__ __forceinline__ const uint8_t *base(int j) const { return j < 8 ? sm.cur : sn.cur; }
  __device__ __forceinline__ uint32_t off(int j) const { return j < 8 ? sm.off[j & 7] : sn.off[j & 7]; }
  __device__ __forceinline__ void frags(uint32_t smem, int wm, int wn, int lane) {
    fa_.init(smem, wm * 128, lane);
    fb_.init(smem + 32768, wn * 128, lane);
  }
  __device__ __forceinline__ void flip(int delta) {
    fa_.flip(delta);
    fb_.flip(delta);
  }
  __device__ __forceinline__ void read(int q, int ks, bf16x8_t (&fa)[NA], bf16x8_t (&fb)[NB]) const {
    if (q == 0) fa[0] = fa_.read(ks, 0);
    else if (q <= NB) fb[q - 1] = fb_.read(ks, q - 1);
    else fa[q - NB] = fa_.read(ks, q - NB);
  }
  __device__ __forceinline__ void store(const BigTile &t, const f32x4_t (&acc)[MI][NI], int wm, int wn,
                                        int lane) const {
    const int M = t.down ? a.f : a.d, N = t.down ? a.d : 2 * a.f;
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      const int n0 = t.n0 + wn * 128 + ni * 16;  // (M and N are multiples of 64: blocks are in or out whole)
      if (n0 >= N) continue;
      bf16 *o = out_row(t, n0 + (lane & 15)) + 16 * ((lane >> 4) & 1) + 8 * (lane >> 5);
#pragma unroll
      for (int j = 0; j < MI / 2; ++j) {
        const int m = t.m0 + wm * 128 + j * 32;
        if (m >= M) continue;
        const f32x4_t x = acc_get(acc[2 * j][ni]), y = acc_get(acc[2 * j + 1][ni]);
        *(uint4 *)(o + m) = pair_rows(make_uint2(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3])),
                                      make_uint2(pk_bf16(y[0], y[1]), pk_bf16(y[2], y[3])));
      }
      __builtin_amdgcn_sched_barrier(0);  // (a block's results at a time, not all 256 in registers)
    }
  }
};

// f(0), f(1), .. f(N - 1) with compile-time arguments
template <int N, class F, int... I>
__device__ __forceinline__ void unroll_(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void unroll(F &&f) {
  unroll_<N>(f, std::make_integer_sequence<int, N>{});
}

// The block's tiles first, first + gridDim.x, .. of problem P; returns P's number of tiles.
template <class P>
__device__ __forceinline__ int big_tiles_run(const MoeGradArgs &a, const BigShape &shape, uint8_t *smem, int first) {
  P p(a, shape);
  constexpr int NM = P::NM, NF = P::NA + P::NB, IPW = P::IPW, STAGE = P::STAGE;
  constexpr int MI = P::MI, NI = P::NI;
  // The schedule of a step, in MFMAs of its two slices of 32: reads of slice 1 beside
  // the first NF of slice 0; a barrier once they are in (after B1J), which frees the
  // stage for the transfers of the stage after the next; before MFMA RS of slice 1 the
  // barrier that publishes the next stage, whose slice 0 is read from there on.
  constexpr int RS = NM - NF < 48 ? NM - NF : 48;
  constexpr int B1J = NF + 2;
  constexpr int NSLOT = (NM - 1 - B1J) + RS;
  constexpr int GAP = NSLOT / IPW < 5 ? NSLOT / IPW : 5;
  static_assert(B1J < NM && RS + NF <= NM && GAP >= 1 && GAP * (IPW - 1) < NSLOT, "room for the transfers");
  const TileScan gs = p.scan();
  const int total = __builtin_amdgcn_readfirstlane(p.total(gs));
  if (first >= total) return total;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
  uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(smem) + wave * 1024);  // the wave's part of the present stage
  int delta = STAGE;                                                             // to the other one
  p.frags(lds_addr(smem), wm, wn, lane);

  // the producer: stage pk of tile Lp; behind the block's last stage the same one again, unused
  int Lp = first - int(gridDim.x), pk = 0, pnk = 0;
  auto advance = [&]() __attribute__((always_inline)) {
    if (pk + 1 < pnk) {
      p.next(++pk);
      return;
    }
    BigTile t;
    int l = Lp;
    do {
      l += int(gridDim.x);
      if (l >= total) return;
      t = p.tile(gs, l, total);
    } while (t.nk == 0);
    Lp = l;
    pk = 0;
    pnk = t.nk;
    p.source(t);
  };
  bf16x8_t fa[2][P::NA], fb[2][P::NB];
  f32x4_t acc[MI][NI];
  advance();
  if (!P::EMPTY || pnk > 0) {  // the block has a product
#pragma unroll
    for (int j = 0; j < IPW; ++j) dma16_s(p.base(j), p.off(j), dst + P::lds_off(j));
    advance();
#pragma unroll
    for (int j = 0; j < IPW; ++j) dma16_s(p.base(j), p.off(j), dst + STAGE + P::lds_off(j));
    advance();
    wait_vm<IPW>();
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NF; ++q) p.read(q, 0, fa[0], fb[0]);
  }
  auto step = [&](auto first) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(first)::value;
    unroll<NM>([&](auto J) __attribute__((always_inline)) {
      constexpr int j = decltype(J)::value, mi = j / NI, ni = j % NI, pos = j - B1J - 1;
      if constexpr (pos >= 0 && pos % GAP == 0 && pos / GAP < IPW)
        mfma_dma<FIRST, P::lds_off(pos / GAP)>(acc[mi][ni], fa[0][mi], fb[0][ni],
                                               p.base(pos / GAP), p.off(pos / GAP), dst);
      else if constexpr (FIRST)
        mfma_agpr_first(acc[mi][ni], fa[0][mi], fb[0][ni]);
      else
        mfma_agpr(acc[mi][ni], fa[0][mi], fb[0][ni]);
      if constexpr (j < NF) p.read(j, 1, fa[1], fb[1]);
      if constexpr (j == B1J) __syncthreads();  // every wave's reads of the stage are in
    });
    p.flip(delta);
    unroll<NM>([&](auto J) __attribute__((always_inline)) {
      constexpr int j = decltype(J)::value, mi = j / NI, ni = j % NI, pos = NM - 1 - B1J + j;
      if constexpr (j == RS) {
        wait_vm<IPW>();  // the next stage is in: only the one after it may be out
        __syncthreads();
      }
      if constexpr (j < RS && pos % GAP == 0 && pos / GAP < IPW)
        mfma_dma<false, P::lds_off(pos / GAP)>(acc[mi][ni], fa[1][mi], fb[1][ni],
                                               p.base(pos / GAP), p.off(pos / GAP), dst);
      else
        mfma_agpr(acc[mi][ni], fa[1][mi], fb[1][ni]);
      if constexpr (j >= RS && j - RS < NF) p.read(j - RS, 0, fa[0], fb[0]);
    });
    dst += delta;
    delta = -delta;
    advance();
  };
  for (int L = first; L < total; L += int(gridDim.x)) {
    const BigTile t = p.tile(gs, L, total);
    if constexpr (P::EMPTY) {
      if (t.nk == 0) {  // an expert without rows
        p.store_zero(t);
        continue;
      }
    }
    step(std::true_type{});
    for (int k = 1; k < t.nk; ++k) step(std::false_type{});
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int i = 0; i < MI; ++i) acc_fence_row<NI>(acc[i]);
    // (an opaque copy of the lane: address terms hoisted out of the tile loop would hold
    // registers through the products)
    int ln = lane;
    asm volatile("" : "+v"(ln));
    p.store(t, acc, wm, wn, ln);
    // the next stage's slice 0 again: its registers served the results
#pragma unroll
    for (int q = 0; q < NF; ++q) p.read(q, 0, fa[0], fb[0]);
  }
  wait_vm<0>();  // (the unused stages)
  return total;
}

// P's tiles, then Q's (which wait for none of P's): the blocks that P leaves a tile short begin Q's
// list, so that the two lose one last round together (160M, 16384 tokens: dn 1.4 rounds and weights
// 2.3: 488 us one after the other, 409 together; 410M, 4000 tokens, skewed: 286 and 238; the fastest of
// ten calls each, of which the means together are 465 and 253).
template <class P, class Q = void>
__global__ __launch_bounds__(256, 1) void moe_grad_big_kernel(MoeGradArgs a, BigShape shape) {
  __shared__ __align__(1024) uint8_t smem[2 * P::STAGE];
  const int n = big_tiles_run<P>(a, shape, smem, blockIdx.x);
  if constexpr (!std::is_void<Q>::value) {
    static_assert(P::STAGE == Q::STAGE, "one array of stages");
    __syncthreads();
    const int g = int(gridDim.x), r = (int(blockIdx.x) - n % g + g) % g;
    big_tiles_run<Q>(a, shape, smem, r);
  }
}

// ------------------------------------------------------------------ tokens
// dn of a token = the sum of its slots' rows of Y; through the norm to dxt; the
// block's share of dg2 (fp32 over the tokens of a block, joined in fp64);
// beside them, in blocks of their own, g_gate from the hidden tiles' partial sums (160M, 1 token:
// 8.1 us after the token's own work, 6.4 beside it).  One wave per token at a time;
// rows of up to 512 RR elements are read once and stay in registers (RR 0: any
// width, read twice).  ONE: dn's sum is not split; without the registers of the parts'
// loads two more waves a SIMD (160M, 16384 tokens 66 us, 50).  Bound by HBM: 1.3B, 16384
// tokens, 453 MB, 127 us (1024 blocks 132; a slot's whole row in flight 135).
constexpr int TOK_BLOCKS = 512;
template <typename T, int RR, bool ONE>
__global__ __launch_bounds__(256) void moe_grad_token_kernel(
    const T *__restrict__ x, const T *dx, const T *__restrict__ g, const float *__restrict__ Y,
    const int32_t *__restrict__ eidx, const int32_t *__restrict__ row_of,
    const int32_t *__restrict__ yrow_of, int planes, int64_t plane, const float *__restrict__ gpart, int GP,
    int N, int k, int d, float eps, T *dxt, float *__restrict__ g_gate, float *__restrict__ part,
    T *__restrict__ dg2, int tb) {
  constexpr int RN = RR > 0 ? RR : 1, PU = ONE ? 1 : 8;
  __shared__ __align__(16) float red[RR > 0 ? 4 : 1][RR > 0 ? 512 * RR : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (int(blockIdx.x) >= tb) {  // the gates' blocks: one wave per assignment
    const int stride = (int(gridDim.x) - tb) * 4;
    for (int64_t i = (int(blockIdx.x) - tb) * 4 + wave; i < int64_t(N) * k; i += stride) {
      float v = 0.f;
      if (eidx[i] != 0)
        for (int j = lane; j < GP; j += 64) v += gpart[int64_t(row_of[i]) * GP + j];
      v = wave_sum(v);
      if (lane == 0) g_gate[i] = v;
    }
    return;
  }
  float sum[RN][8];  // the wave's share of dg2
#pragma unroll
  for (int q = 0; q < RN; ++q)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[q][j] = 0.f;
  // (RR 0: every wave has a row of part and adds to it)
  float *pr = RR == 0 && part ? part + (int64_t(blockIdx.x) * 4 + wave) * d : nullptr;
  if (RR == 0 && pr)
    for (int c = lane * 8; c < d; c += 512) store8(pr + c, &sum[0][0]);
  for (int i = blockIdx.x * 4 + wave; i < N; i += tb * 4) {
    const T *xr = x + int64_t(i) * d;
    const int32_t *ei = eidx + int64_t(i) * k, *yo = yrow_of + int64_t(i) * k;
    auto dn8 = [&](int c, float *dn) {
#pragma unroll
      for (int j = 0; j < 8; ++j) dn[j] = 0.f;
      for (int s = 0; s < k; ++s) {
        if (ei[s] == 0) continue;
        const float *yr = Y + int64_t(yo[s]) * d + c;
        // the parts of a split sum, in order, eight loads in flight
        for (int p0 = 0; p0 < (ONE ? 1 : planes); p0 += PU) {
          float y[PU][8];
#pragma unroll
          for (int p = 0; p < PU; ++p)
            if (p == 0 || p0 + p < planes) load8(yr + (p0 + p) * plane, y[p]);
#pragma unroll
          for (int p = 0; p < PU; ++p)
            if (p == 0 || p0 + p < planes) {
#pragma unroll
              for (int j = 0; j < 8; ++j) dn[j] += y[p][j];
            }
        }
      }
    };
    float w[RN][8], dn[RN][8], up[RN][8];
    double ss = 0.0, dot = 0.0;
    auto take = [&](int c, float *wv, float *dv, float *uv) {  // the sums over a row
      float gv[8];
      load8(xr + c, wv);
      load8(g + c, gv);
      if constexpr (RR > 0) load8(dx + int64_t(i) * d + c, uv);
      dn8(c, dv);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ss = fma(double(wv[j]), double(wv[j]), ss);
        dot = fma(double(dv[j] * gv[j]), double(wv[j]), dot);
      }
    };
    if constexpr (RR > 0) {
#pragma unroll
      for (int q = 0; q < RN; ++q)
        if (lane * 8 + 512 * q < d) take(lane * 8 + 512 * q, w[q], dn[q], up[q]);
    } else {
      for (int c = lane * 8; c < d; c += 512) take(c, w[0], dn[0], up[0]);
    }
    ss = wave_sum(ss);
    dot = wave_sum(dot);
    const double r = 1.0 / sqrt(ss / double(d) + double(eps));
    const float rf = float(r), cf = float(r * r * r * dot / double(d));
    auto give = [&](int c, const float *wv, const float *dv, const float *u, float *q) {
      float gv[8], o[8];
      load8(g + c, gv);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = u[j] + fmaf(rf, dv[j] * gv[j], -cf * wv[j]);
        q[j] = fmaf(dv[j] * rf, wv[j], q[j]);
      }
      store8(dxt + int64_t(i) * d + c, o);
    };
    if constexpr (RR > 0) {
#pragma unroll
      for (int q = 0; q < RN; ++q)
        if (lane * 8 + 512 * q < d) give(lane * 8 + 512 * q, w[q], dn[q], up[q], sum[q]);
    } else {
      for (int c = lane * 8; c < d; c += 512) {
        float q[8];
        load8(xr + c, w[0]);
        load8(dx + int64_t(i) * d + c, up[0]);
        dn8(c, dn[0]);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = 0.f;
        if (pr) load8(pr + c, q);
        give(c, w[0], dn[0], up[0], q);
        if (pr) store8(pr + c, q);
      }
    }
  }
  if constexpr (RR > 0) {
    if (!part && !dg2) return;
#pragma unroll
    for (int q = 0; q < RN; ++q) store8(&red[wave][512 * q + lane * 8], sum[q]);
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += 256) {
      const float v = ((red[0][c] + red[1][c]) + red[2][c]) + red[3][c];
      if (dg2)  // (the only block)
        Act<T>::st(dg2, c, v);
      else
        part[int64_t(blockIdx.x) * d + c] = v;
    }
  }
}

// dg2 from the token blocks' rows of partial sums: 16 columns a block, 64 threads a
// column over the rows, joined in fp64 in a fixed order.
template <typename T>
__global__ __launch_bounds__(1024) void moe_grad_g2_kernel(const float *__restrict__ part, int rows, int d,
                                                           T *__restrict__ dg2) {
  __shared__ double red[64][17];
  const int col = threadIdx.x & 15, at = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  constexpr int U = 8;
  double v = 0.0;
  for (int r0 = at; r0 < rows; r0 += 64 * U) {
    float t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) t[u] = r0 + 64 * u < rows ? part[int64_t(r0 + 64 * u) * d + c] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) v += double(t[u]);
  }
  red[at][col] = v;
  __syncthreads();
  if (at < 8) {
    v = red[at][col];
#pragma unroll
    for (int j = 1; j < 8; ++j) v += red[at + 8 * j][col];
    red[at][col] = v;
  }
  __syncthreads();
  if (at == 0) {
#pragma unroll
    for (int j = 1; j < 8; ++j) v += red[j][col];
    Act<T>::st(dg2, c, float(v));
  }
}

// ------------------------------------------------------------------ launchers
static int cu_count() {
  static const int n = [] {
    int dev = 0, v = 0;
    return hipGetDevice(&dev) == hipSuccess &&
                   hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0
               ? v
               : 256;
  }();
  return n;
}

int moe_grad_gate_parts(const triroute_cfg &cfg) { return cfg.d_ff / 64 * 2; }
static int token_blocks(int N) { return std::min((N + 3) / 4, TOK_BLOCKS); }
int moe_grad_part_rows(const triroute_cfg &cfg, int N) {
  return token_blocks(N) * (cfg.d_model <= 2048 ? 1 : 4);
}

// bf16: whether the 256 x 256 tiles serve: where an expert has r >= 96 rows (when the router
// spreads its options evenly), so that a tile is not mostly padding, and q's tiles, the fewest, give
// each of the 256 CUs one.  Us, small tiles / large ones.  By tiles, T: 160M, T 192 225 / 249 and
// 247 / 249, T 256 281 / 261 and 319 / 275; 410M, T 176 312 / 339, T 264 382 / 399, T 352
// 490 / 437; 2048 x 5632, one expert, T 88 276 / 410, four, T 176 545 / 609; 256 x 512, four, T 104
// 137 / 146, T 416 572 / 498; 512 x 1024, eight, T 256 240 / 208.  By r: 1.3B (T 352), r 32
// 740 / 859, r 64 910 / 940, r 96 970 / 993, r 256 1582 / 1221; 63 experts of 768 x 2048, r 64
// 509 / 504, r 128 653 / 580; of 2048 x 5632, r 32 2680 / 2850, r 64 3241 / 3084.
static bool big_tiles(const triroute_cfg &cfg, int N) {
  const int64_t r = int64_t(N) * cfg.top_k / (cfg.n_experts + 1);
  return cfg.act == TRIROUTE_BF16 && r >= 96 &&
         cfg.n_experts * ((r + 255) / 256) * ((cfg.d_ff + 255) / 256) >= 256;
}
// Parts of the sum of dn for few rows, so that the stream of the weights has about
// two blocks a CU: at most 8 (a token's partial rows are loaded together), each of at least 4 blocks of 64 units
// (fp32, whose steps are half as long: 2; the small layer, 128 tokens: dn 14.6 -> 8.9 us with
// four parts instead of two; 160M, 1 token, bf16: 16 parts of 2 blocks gain nothing there and cost the
// tokens 3 us).
int moe_grad_splits(const triroute_cfg &cfg, int N) {
  if (big_tiles(cfg, N)) return 1;
  const int Nk = N * cfg.top_k;
  const int64_t tiles = int64_t(Nk / INP_R + std::min(cfg.n_experts, Nk)) * (cfg.d_model / INP_M);
  return std::max(1, std::min({int((512 + tiles - 1) / tiles), cfg.d_ff / 64 / (cfg.act == TRIROUTE_BF16 ? 4 : 2), 8}));
}

template <typename T>
static hipError_t backward(const triroute_cfg &cfg, int N, const MoeGradJob &j, hipStream_t st) {
  const int E = cfg.n_experts, k = cfg.top_k, d = cfg.d_model, f = cfg.d_ff, Nk = N * k;
  const int64_t rows = moe_grad_rows(cfg, N);
  MoeGradArgs a;
  a.Wg = j.w.Wgate; a.Wu = j.w.Wup; a.Wd = j.w.Wdown;
  a.n2 = j.n2; a.dy = j.dy; a.dGU = j.dGU;
  a.Hp = j.out.dWgate ? j.Hp : nullptr;
  a.gate = j.gate; a.Y = j.Y; a.gpart = j.gpart;
  a.dWg = j.out.dWgate; a.dWu = j.out.dWup; a.dWd = j.out.dWdown;
  a.cnt = j.cmp.exp_cnt;
  a.E = E; a.d = d; a.f = f;
  a.GP = moe_grad_gate_parts(cfg);
  moe_grad_rows_kernel<T><<<unsigned(std::min<int64_t>((rows + 3) / 4, ROW_BLOCKS)), 256, 0, st>>>(
      (const T *)j.xt, (const T *)j.dx, (const T *)j.g2, j.egate, j.cmp.exp_cnt, j.cmp.exp_rows, E, k, d,
      cfg.rms_eps, (T *)j.n2, (T *)j.dy, j.gate, j.row_of, j.list_of);
  const int32_t *yrow_of = j.row_of;
  int splits = 1;
  bool done = false;
  const int64_t plane = int64_t(Nk) * d;
  if constexpr (sizeof(T) == 2) {
    if (big_tiles(cfg, N)) {
      const int cu = cu_count();
      a.GP = f / 64;
      BigShape sh{};
      sh.md = (d + 255) / 256;
      sh.mf = (f + 255) / 256;
      sh.t1 = sh.md * ((2 * f + 255) / 256);
      sh.t2 = sh.md * sh.mf;
      auto blocks = [&](int ny) { return unsigned(std::min<int64_t>((int64_t(Nk) / 256 + E) * ny, cu)); };
      sh.ny = sh.mf;
      moe_grad_big_kernel<RowsBig<false>><<<blocks(sh.ny), 256, 0, st>>>(a, sh);
      sh.ny = (f + 127) / 128;
      moe_grad_big_kernel<GateUpBig><<<blocks(sh.ny), 256, 0, st>>>(a, sh);
      sh.ny = sh.md;
      if (a.Hp)
        moe_grad_big_kernel<RowsBig<true>, WeightBig><<<cu, 256, 0, st>>>(a, sh);
      else
        moe_grad_big_kernel<RowsBig<true>><<<blocks(sh.ny), 256, 0, st>>>(a, sh);
      done = true;
    }
  }
  if (!done) {
    const int nf = f / 64, nd = d / INP_M, rt = Nk / 64 + std::min(E, Nk);  // row tiles at most
    splits = moe_grad_splits(cfg, N);
    yrow_of = j.list_of;
    if (int64_t(rt) * nf * 2 <= cu_count())
      moe_grad_hidden_kernel<T, 32, 4><<<unsigned(rt) * nf * 2, 512, 0, st>>>(a, nf * 2);
    else if (int64_t(rt) * nf <= cu_count())
      moe_grad_hidden_kernel<T, 64, 3><<<unsigned(rt) * nf, 512, 0, st>>>(a, nf);
    else
      moe_grad_hidden_kernel<T, 64, 2><<<unsigned(rt) * nf, 512, 0, st>>>(a, nf);
    const unsigned nin = unsigned(rt) * nd * splits;
    if (a.Hp) {
      const int md = (d + WGT_T - 1) / WGT_T, mf = (f + WGT_T - 1) / WGT_T;
      const unsigned tiles = unsigned(E) * (md * (2 * f / WGT_T) + mf * md);
      moe_grad_input_weight_kernel<T><<<nin + tiles, 256, 0, st>>>(a, int(nin), nd, splits, plane);
    } else {
      moe_grad_input_kernel<T><<<nin, 256, 0, st>>>(a, nd, splits, plane);
    }
  }
  const int prows = moe_grad_part_rows(cfg, N), tb = token_blocks(N);
  const bool direct = tb == 1 && d <= 2048;  // one block: its dg2 is the sum
  const unsigned blocks = tb + (j.out.g_gate ? std::min((Nk + 3) / 4, TOK_BLOCKS) : 0);
  auto launch = [&](auto rr, auto one) {
    moe_grad_token_kernel<T, decltype(rr)::value, decltype(one)::value><<<blocks, 256, 0, st>>>(
        (const T *)j.xt, (const T *)j.dx, (const T *)j.g2, j.Y, j.eidx, j.row_of, yrow_of, splits, plane, j.gpart,
        a.GP, N, k, d, cfg.rms_eps, (T *)j.out.dxt, j.out.g_gate, j.out.dg2 && !direct ? j.part : nullptr,
        direct ? (T *)j.out.dg2 : nullptr, tb);
  };
  auto token = [&](auto rr) {
    if (splits == 1) launch(rr, std::true_type{});
    else launch(rr, std::false_type{});
  };
  if (d <= 512) token(std::integral_constant<int, 1>{});
  else if (d <= 1024) token(std::integral_constant<int, 2>{});
  else if (d <= 2048) token(std::integral_constant<int, 4>{});
  else token(std::integral_constant<int, 0>{});
  if (j.out.dg2 && !direct)
    moe_grad_g2_kernel<T><<<d / 16, 1024, 0, st>>>(j.part, prows, d, (T *)j.out.dg2);
  return hipGetLastError();
}

hipError_t launch_moe_backward(const triroute_cfg &cfg, int N, const MoeGradJob &j, hipStream_t st) {
  return cfg.act == TRIROUTE_BF16 ? backward<bf16>(cfg, N, j, st) : backward<float>(cfg, N, j, st);
}

}  // namespace tr
