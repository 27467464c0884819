// The two MFMA product kernels, C = A B^T with both operands K-contiguous, and the
// choice of their tiles: gemm_mfma_kernel, BM x BN tiles on WM x WN waves with S
// operand stages in LDS, for few and middling rows, and the persistent four-wave
// gemm_w4_kernel for many.  The launchers choose the tile by the rounds it makes
// over the CUs.  A problem P names its operands' type (P::Op: bf16 with fp32 sums, or
// 8-bit codes with int32 sums), its rows and its epilogue.  K counts two-byte units of an
// operand row (a bf16 element, a pair of codes): a product of as many bytes takes the
// same stages, fragments and MFMA cycles in either type.
#pragma once

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "gemm_tile.hpp"
#include "kernels.hpp"

namespace tr {

struct MTile {
  int m0, n0, mvalid, e, p0;
  int k0 = 0, yp = 0;  // K offset of a split product and its output plane
};

// Row tiles of the grouped problems: lane e - 1 of every wave holds expert
// e's row count and tile count, and an inclusive scan over the lanes gives
// the tiles of experts 1..e, so the mapping costs one parallel load instead
// of a chain of E dependent ones (E <= 63).
struct GroupScan {
  int c = 0, nt = 0, incl = 0, total = 0, start = 0;
};

__device__ __forceinline__ GroupScan group_scan(int BM, const int32_t *cnt, int E) {
  const int lane = threadIdx.x & 63;
  GroupScan g;
  g.c = lane < E ? cnt[lane + 1] : 0;
  g.nt = (g.c + BM - 1) / BM;
  int x = g.nt;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  g.incl = x;
  g.total = __shfl(x, 63, 64);
  // first list position of expert lane + 1: the lists lie back to back in
  // expert order, so it is the sum of the counts before it
  int s = g.c;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(s, d, 64);
    if (lane >= d) s += y;
  }
  g.start = s - g.c;
  return g;
}

// Map a linear row-tile index to (expert e >= 1, tile within e).
__device__ __forceinline__ bool mmap_grouped(int bx, int BM, const GroupScan &gs, MTile &t) {
  const uint64_t m = __ballot(gs.incl > bx);
  if (!m) return false;
  const int l = __ffsll((unsigned long long)m) - 1;
  const int incl = __shfl(gs.incl, l, 64), nt = __shfl(gs.nt, l, 64), c = __shfl(gs.c, l, 64);
  const int rem = bx - (incl - nt);
  t.e = l + 1;
  t.p0 = __shfl(gs.start, l, 64) + rem * BM;
  t.mvalid = min(BM, c - rem * BM);
  t.m0 = 0;
  return true;
}

// Physical column n of a BN-wide tile -> (pair index P in the tile, half).
// Wave slice s = n / 64 holds pairs 32 s .. 32 s + 31: first halves in its
// columns 0..31, second halves in 32..63.
__device__ __forceinline__ void col_pair(int n, int &P, int &half) {
  P = (n >> 6) * 32 + (n & 31);
  half = (n >> 5) & 1;
}

// ---------------------------------------------------------------- problems
// Each problem names its operand rows (a_row, b_row), the LDS column of an
// accumulator after the register pass (EPI_ROPE / EPI_SWIGLU combine the
// partner columns first), and a row-wise epilogue that reads the staged fp32
// tile C (NC columns, row stride LDC) and writes 16-byte chunks.
enum { EPI_PLAIN = 0, EPI_ROPE = 1, EPI_SWIGLU = 2 };

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

__device__ __forceinline__ u32x4_t pack8_bf16(const float *v) {
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pk_bf16(v[2 * i], v[2 * i + 1]);
  return w;
}

// ------------------------------------------------------------------ kernel
// The same within each expert of a grouped problem: tile t lies in the
// first expert whose tiles (row tiles x ny, in expert order) reach past it.
__device__ __forceinline__ void grouped_band_order(int t, int ny, const GroupScan &gs, int &bx,
                                                   int &by) {
  const uint64_t m = __ballot(gs.incl * ny > t);
  const int l = __ffsll((unsigned long long)m) - 1;
  const int nt = __shfl(gs.nt, l, 64), first = __shfl(gs.incl, l, 64) - nt;
  int i;
  band_order(t - first * ny, nt, ny, i, by);
  bx = first + i;
}

// Epilogue register pass: lane holds rows 4 (lane/16) + i of each 16-row tile
// and column (lane % 16) of each 16-column block; in each 64-column slice the
// partner columns (ni, ni + 2) are combined for SwiGLU and kept apart for
// RoPE.  The problem's row-wise pass then reads the staged fp32 tile C.
template <class P, int MI, int NI, int TM, int TN, int LDC>
__device__ __forceinline__ void store_acc(const P &p, float *C, const f32x4_t (&acc)[MI][NI],
                                          int wm, int wn, int lane) {
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wm * TM + mi * 16 + 4 * (lane >> 4) + i;
      if constexpr (P::EPI == EPI_PLAIN) {
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
          C[r * LDC + wn * TN + ni * 16 + (lane & 15)] = acc[mi][ni][i];
      } else {
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
          if ((ni & 3) >= 2) continue;
          int Pp, half;
          col_pair(wn * TN + ni * 16 + (lane & 15), Pp, half);
          const float g = acc[mi][ni][i], u = acc[mi][ni + 2][i];
          if constexpr (P::EPI == EPI_SWIGLU) {
            C[r * LDC + Pp] = g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u;
          } else {
            C[r * LDC + p.ccol(Pp, 0)] = g;
            C[r * LDC + p.ccol(Pp, 1)] = u;
          }
        }
      }
    }
}

// KW > 1: the block holds KW groups of WM x WN waves, each with its own stages
// over a KW-th of K; the partial tiles are added in group order at the end.
// A few rows against a small weight give one block a CU at most, which walks
// K in a chain of round trips to memory; KW groups make the chain that much
// shorter.
template <class P, int BM, int BN, int WM, int WN, int BK, int S, int KW>
__global__ __launch_bounds__(64 * WM * WN * KW, 1) void gemm_mfma_kernel(P p, int K, int ny) {
  typedef typename P::Op Op;
  constexpr int NW = WM * WN, NT = 64 * NW * KW;  // waves of a K group, threads
  constexpr int TM = BM / WM, TN = BN / WN;  // wave tile
  constexpr int MI = TM / 16, NI = TN / 16;  // 16 x 16 MFMA tiles per wave
  constexpr int RB = BK * 2;                 // bytes per operand row per K step
  constexpr int CPR = RB / 16;               // 16-byte chunks per row
  constexpr int RPT = 1024 / RB;             // rows per 1 KB transfer
  constexpr int STAGE = (BM + BN) * RB;
  constexpr int IPW = STAGE / 1024 / NW;     // 1 KB transfers per wave per stage
  static_assert(STAGE % (1024 * NW) == 0 && TN % 64 == 0, "whole transfers, 64-column slices");
  static_assert(S >= 2 && S <= 6 && (BK == 32 || BK == 64), "pipeline shape");
  constexpr int NC = P::out_cols(BN), LDC = NC + 16;  // staged output tile (fp32)
  constexpr int PART = BM * BN * 4;                    // a group's partial tile
  constexpr int OUT = BM * LDC * 4 > (KW - 1) * PART ? BM * LDC * 4 : (KW - 1) * PART;
  constexpr int SMEM = KW * S * STAGE > OUT ? KW * S * STAGE : OUT;
  __shared__ __align__(1024) uint8_t smem_all[SMEM];
  GroupScan gs;
  if constexpr (P::GROUPED) gs = group_scan(BM, p.cnt, p.E);
  const int total = p.tiles(BM, ny, gs);
  if (int(blockIdx.x) >= total) return;
  const int t = xcd_tile(blockIdx.x, total);
  MTile tc;
  if (!p.map(t / ny, t % ny, BM, BN, tc, gs)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int kg = KW > 1 ? (tid >> 6) / NW : 0, wave = KW > 1 ? (tid >> 6) % NW : tid >> 6;
  const int wm = wave / WN, wn = wave % WN;
  uint8_t *smem = smem_all + kg * S * STAGE;  // the group's stages
  // its K steps, from step kg nk on; of 8-bit operands the last groups may have fewer
  constexpr bool UNEVEN = Op::INT && KW > 1;
  const int nk = UNEVEN ? (K / BK + KW - 1) / KW : K / BK / KW;
  const int own = UNEVEN ? max(min(nk, K / BK - kg * nk), 0) : nk;
  // Transfer j of this wave fills stage rows RPT g .. RPT g + RPT - 1
  // (g = wave IPW + j; A rows first, then B rows).  Lane l writes LDS chunk
  // l % CPR of row RPT g + l / CPR, which holds the source chunk that swz
  // maps there.  Rows past the valid rows (or past the weight's columns)
  // read a valid row instead: their products land in accumulator rows /
  // columns the epilogue never stores.
  const uint8_t *src[IPW];
  const auto *b_fallback = p.b_row(tc, 0);
#pragma unroll
  for (int j = 0; j < IPW; ++j) {
    const int rr = RPT * (wave * IPW + j) + lane / CPR;
    const int c = swz<CPR>(rr, lane % CPR);  // swz is an involution in c
    const typename Op::elem *row;
    if (rr < BM) {
      row = p.a_row(tc, rr < tc.mvalid ? rr : 0);
    } else {
      row = p.b_row(tc, rr - BM);
      if (!row) row = b_fallback;
    }
    src[j] = (const uint8_t *)row + c * 16 + kg * nk * RB;
  }
  const uint32_t sbase = lds_addr(smem) + wave * IPW * 1024;
  auto issue = [&](int kt, int stage) {
#pragma unroll
    for (int j = 0; j < IPW; ++j) dma16(src[j] + kt * RB, sbase + stage * STAGE + j * 1024);
  };
  typename Op::acc acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = typename Op::acc{0, 0, 0, 0};
#pragma unroll
  for (int s0 = 0; s0 < S - 1; ++s0)
    if (s0 < own) issue(s0, s0);
  for (int kt = 0; kt < nk; ++kt) {
    // stage kt has landed once at most the later stages' transfers are out
    wait_stages<IPW, S>(min(S - 2, own - 1 - kt));
    __syncthreads();  // every wave's part of stage kt is in; stage kt-1 is free
    if (kt + S - 1 < own) issue(kt + S - 1, (kt + S - 1) % S);
    if (UNEVEN && kt >= own) continue;  // (the barriers are all groups')
    const uint8_t *As = smem + (kt % S) * STAGE;
    const uint8_t *Bs = As + BM * RB;
#pragma unroll
    for (int ks = 0; ks < BK / 32; ++ks) {
      const int ch = ks * 4 + (lane >> 4);
      typename Op::frag b[NI];
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) {
        const int n = wn * TN + ni * 16 + (lane & 15);
        b[ni] = *(const typename Op::frag *)(Bs + n * RB + (swz<CPR>(n, ch) << 4));
      }
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int r = wm * TM + mi * 16 + (lane & 15);
        const typename Op::frag a = *(const typename Op::frag *)(As + r * RB + (swz<CPR>(r, ch) << 4));
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
          acc[mi][ni] = Op::mma(a, b[ni], acc[mi][ni]);
      }
    }
  }
  __syncthreads();  // every wave is done with the operand stages
  float *C = (float *)smem_all;
  if constexpr (KW > 1) {
    // partial tiles of groups 1 .. KW - 1, [group][wave][register][lane]
    typedef typename Op::sum sum_t;  // (fp32 or int32: four bytes)
    sum_t *part = (sum_t *)smem_all + wave * (PART / 4 / NW) + lane;
    if (kg > 0) {
      sum_t *o = part + (kg - 1) * (PART / 4);
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[((mi * NI + ni) * 4 + i) * 64] = acc[mi][ni][i];
    }
    __syncthreads();
    if (kg == 0) {
#pragma unroll
      for (int g = 0; g < KW - 1; ++g)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
          for (int ni = 0; ni < NI; ++ni)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[mi][ni][i] += part[g * (PART / 4) + ((mi * NI + ni) * 4 + i) * 64];
    }
    __syncthreads();
  }
  if (KW == 1 || kg == 0) {
    if constexpr (Op::INT)
      p.template stage<MI, NI, TM, TN, LDC>(tc, C, acc, wm, wn, lane);
    else
      store_acc<P, MI, NI, TM, TN, LDC>(p, C, acc, wm, wn, lane);
  }
  __syncthreads();
  p.template epilogue<BM, NC, LDC, NT>(tc, C, tid);
}

// ------------------------------------------------------- four-wave kernel
// One wave per SIMD, each wave a (BM/2) x (BN/2) sub-tile: every operand byte
// read from LDS feeds twice the MFMAs of a 128 x 64 wave tile (per K
// step and CU, 128 KB of fragment reads against 256 MFMAs per SIMD).  With
// no second wave on its SIMD to switch to, a wave hides LDS latency itself:
// the fragments of the next 32-wide K slice are read into a second register
// set while the current slice's MFMAs issue, the reads slotted between the
// MFMAs.  Stages are double-buffered (BK = 64); stage kt + 2 goes into the
// buffer of stage kt as soon as every wave has read it (schedule below).
template <class P, int BM, int BN>
__global__ __launch_bounds__(256, 1) void gemm_w4_kernel(P p, int K, int ny) {
  constexpr int NW = 4, NT = 256, WN = 2;
  constexpr int TM = BM / 2, TN = BN / 2;    // wave tile
  constexpr int MI = TM / 16, NI = TN / 16;  // 16 x 16 MFMA tiles per wave
  constexpr int BK = 64, RB = 128, CPR = 8, RPT = 8;
  constexpr int STAGE = (BM + BN) * RB;
  constexpr int IPW = STAGE / 1024 / NW;  // 1 KB transfers per wave per stage
  constexpr int NF = MI + NI;             // fragment reads per K slice
  constexpr int NM = MI * NI;             // MFMAs per K slice
  static_assert(STAGE % (1024 * NW) == 0 && (TN % 64 == 0 || P::DIRECT_W4), "whole transfers, 64-column slices");
  // K step schedule, two barriers: the first, after MFMA B1J of slice 0
  // (every wave's reads of set 1, the last reads of stage kt, are in), frees
  // the buffer of stage kt; the transfers of stage kt + 2 go out one every GAP
  // MFMAs from there until MFMA RS of slice 1, where the second barrier
  // publishes stage kt + 1 (at most this step's IPW transfers still out) for
  // the reads of set 0.  A transfer thus has from slice 0 of step kt to
  // slice 1 of step kt + 1 to land.  (One barrier 16 MFMAs into slice 1, with
  // the transfers after it, left the last ones under 90 MFMAs to land, and a
  // cache-missing transfer stalled the wave at that barrier; spacing the
  // transfers closer than 5 MFMAs slowed the MFMA issue.)
  constexpr int RS = NM - NF < 48 ? NM - NF : 48;
  constexpr int B1J = NF + 4;
  constexpr int NSLOT = (NM - 1 - B1J) + RS;  // slice 0 after B1J, then slice 1 before RS
  constexpr int GAP = NSLOT / IPW < 5 ? NSLOT / IPW : 5;
  static_assert(B1J < NM && RS >= 16 && RS + NF <= NM && GAP >= 1 && GAP * (IPW - 1) < NSLOT,
                "room for the reads and transfers");
  static_assert(P::DIRECT_W4, "results are written from the accumulators");
  // 8-bit products: the scales of each wave's TM rows and TN columns lie behind the stages.  They
  // come in the tile's first K step, as transfers like the operands' (a load into registers
  // would be waited for behind the next tile's transfers, at the tile's end) ahead of the next
  // stage's, so that step's wait covers them.
  constexpr int NSC = P::Op::INT ? TM + TN : 0;
  __shared__ __align__(1024) uint8_t smem[2 * STAGE + NW * NSC * 4];
  // Persistent: block b takes tiles b, b + gridDim.x, ... (one block per CU).
  // The operand stream runs on across tiles: the last two K steps of a tile
  // fetch the first two stages of the block's next tile, so its transfers
  // are in flight while this one's results are written.
  GroupScan gs;
  if constexpr (P::GROUPED) gs = group_scan(BM, p.cnt, p.E);
  const int total = __builtin_amdgcn_readfirstlane(p.tiles(BM, ny, gs));
  int L = blockIdx.x;
  if (L >= total) return;
  // Grouped 8-bit problems: lane j holds the block's tile j of each 64 (found once, side by side;
  // one after the other, at each tile's end, the search takes 2000 cycles of a tile's 40000 to
  // 70000 there).
  constexpr bool LISTED = P::GROUPED && P::Op::INT;
  MTile mine{};
  auto list_tiles = [&](int first) {
    if constexpr (LISTED) {
      const int l = first + int(gridDim.x) * (threadIdx.x & 63);
      const int x = xcd_tile(min(l, total - 1), total);
      int e = 0, done = 0, incl = 0, start = 0, c = 0;  // the expert whose tiles reach past x
      for (int k = 0; k < p.E; ++k) {
        const int ik = __builtin_amdgcn_readlane(gs.incl, k);
        const bool here = !done && ik * ny > x;
        const int ck = __builtin_amdgcn_readlane(gs.c, k), sk = __builtin_amdgcn_readlane(gs.start, k);
        const int nk = __builtin_amdgcn_readlane(gs.nt, k);
        e = here ? k + 1 : e;
        incl = here ? ik - nk : incl;  // tiles before it
        start = here ? sk : start;
        c = here ? ck : c;
        done |= here;
      }
      int i, j;
      band_order(x - incl * ny, (c + BM - 1) / BM, ny, i, j);
      mine.e = e;
      mine.p0 = start + i * BM;
      mine.mvalid = min(BM, c - i * BM);
      mine.n0 = P::first_unit(j, BN);
    }
  };
  auto tile = [&](int l) {  // a tile's fields are wave-uniform: kept in SGPRs
    MTile t;
    if constexpr (LISTED) {
      const int j = (l - int(blockIdx.x)) / int(gridDim.x);
      if ((j & 63) == 0) list_tiles(l);
      t.m0 = 0;
      t.n0 = __builtin_amdgcn_readlane(mine.n0, j & 63);
      t.mvalid = __builtin_amdgcn_readlane(mine.mvalid, j & 63);
      t.e = __builtin_amdgcn_readlane(mine.e, j & 63);
      t.p0 = __builtin_amdgcn_readlane(mine.p0, j & 63);
      return t;
    }
    const int x = xcd_tile(l, total);
    int bx, by;
    if constexpr (P::GROUPED)
      grouped_band_order(x, ny, gs, bx, by);
    else
      band_order(x, total / ny, ny, bx, by);
    p.map(bx, by, BM, BN, t, gs);  // every index below total maps to a tile
    t.m0 = __builtin_amdgcn_readfirstlane(t.m0);
    t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
    t.mvalid = __builtin_amdgcn_readfirstlane(t.mvalid);
    t.e = __builtin_amdgcn_readfirstlane(t.e);
    t.p0 = __builtin_amdgcn_readfirstlane(t.p0);
    return t;
  };
  MTile tc = tile(L), tn = tc;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // wave-uniform, in SGPRs
  const int wm = wave / WN, wn = wave % WN;
  // Transfer j of this wave fills stage rows RPT (wave IPW + j) .. + RPT - 1
  // as in the kernel above.  A transfer's rows are all A rows or all B
  // rows (RPT divides BM), so each lane keeps one 32-bit byte offset per
  // transfer from that operand's base (the host checks that every operand
  // row lies within 4 GB of it); the base moves on by 128 B per K step.
  // Rows past the valid ones read a valid row instead: their products land
  // in accumulators that are never stored.
  static_assert(BM % RPT == 0, "a transfer stays within one operand");
  auto is_a = [&](int j) { return RPT * (wave * IPW + j) < BM; };  // wave-uniform
  // 8-bit problems: matrices may lie far apart, and a transfer's B rows lie in one of two
  // (P::b_pick of the transfer), whose bases follow the tile: now, and the step to the next tile's.
  uint64_t bnow[2] = {0, 0}, bstep[2] = {0, 0};
  auto base_of = [&](const MTile &t, auto k) -> uint64_t {
    if constexpr (P::Op::INT) {
      const int n = max(RPT * wave * IPW - BM, 0);  // the wave's first B row
      return uint64_t(p.template b_base_w4<TN, decltype(k)::value>(t.n0, n / TN));
    }
    return 0;
  };
  std::integral_constant<int, 0> K0;
  std::integral_constant<int, 1> K1;
  bnow[0] = base_of(tc, K0);
  bnow[1] = base_of(tc, K1);
  auto gbase = [&](int j, bool next) {
    if constexpr (P::Op::INT) {
      const uint64_t b = P::b_pick(j) ? bnow[1] + (next ? bstep[1] : 0) : bnow[0] + (next ? bstep[0] : 0);
      return is_a(j) ? (const uint8_t *)p.a_base() : (const uint8_t *)b;
    } else {
      return (const uint8_t *)(is_a(j) ? p.a_base() : p.b_base());
    }
  };
  // (lane-derived terms of the per-tile address arithmetic start from an
  // opaque copy of the lane: hoisted out of the tile loop they would hold
  // registers through the K loop)
  auto pinned_lane = [&]() {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    return ln;
  };
  auto offsets = [&](const MTile &t, uint32_t(&o)[IPW]) {
    const int ln = pinned_lane();
#pragma unroll
    for (int j = 0; j < IPW; ++j) {
      const int rr = RPT * (wave * IPW + j) + ln / CPR;
      const uint32_t c16 = swz<CPR>(rr, ln % CPR) * 16;
      if (is_a(j))
        o[j] = p.a_off(t, rr < t.mvalid ? rr : 0) + c16;
      else
        o[j] = p.template b_off_w4<NI>(t, (rr - BM) / TN, ((rr - BM) % TN) >> 4, (rr - BM) & 15) + c16;
    }
  };
  uint32_t voff[IPW], vnx[IPW];
  offsets(tc, voff);
  const uint32_t sbase = lds_addr(smem) + wave * IPW * 1024;
  // Fragment addresses: row r = (wave row) + 16 i + lane % 16 reads chunk
  // (4 ks + lane / 16) ^ ((r >> 1) & 7); the XOR term depends on the lane only.
  const int l15 = lane & 15, x7 = (lane >> 1) & 7;
  const uint8_t *fa0 = smem + (wm * TM + l15) * RB;
  const uint8_t *fb0 = smem + BM * RB + (wn * TN + l15) * RB;
  int coff[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) coff[ks] = (((ks * 4 + (lane >> 4)) ^ x7) << 4);

  typedef typename P::Op::frag frag;
  frag fa[2][MI], fb[2][NI];
  // piece q of slice ks in buffer buf: q = 0 is A0, 1..NI the B pieces, then A1..
  auto read_piece = [&](int set, int buf, int q) {
    if (q == 0) {
      fa[set][0] = *(const frag *)(fa0 + buf * STAGE + coff[set]);
    } else if (q <= NI) {
      fb[set][q - 1] = *(const frag *)(fb0 + buf * STAGE + (q - 1) * 16 * RB + coff[set]);
    } else {
      const int mi = q - NI;
      fa[set][mi] = *(const frag *)(fa0 + buf * STAGE + mi * 16 * RB + coff[set]);
    }
  };
  typename P::Op::acc acc[MI][NI];
  auto mma = [&](int set, int j) {
    mfma_agpr(acc[j / NI][j % NI], fa[set][j / NI], fb[set][j % NI]);
  };
  auto mma_first = [&](int set, int j) {
    mfma_agpr_first(acc[j / NI][j % NI], fa[set][j / NI], fb[set][j % NI]);
  };

  auto issue_scales = [&](const MTile &t) {
    if constexpr (P::Op::INT) {
      const uint32_t at = lds_addr(smem) + 2 * STAGE + wave * NSC * 4;
      const int ln = pinned_lane();
#pragma unroll
      for (int j = 0; j < TM / 64; ++j) {
        const int r = wm * TM + 64 * j + ln;
        dma4(p.row_scale_at(t, r < t.mvalid ? r : 0), at + j * 256);
      }
#pragma unroll
      for (int j = 0; j < TN / 64; ++j)
        dma4(p.template col_scale_at<TN>(t, wn, 64 * j + ln), at + (TM + 64 * j) * 4);
    }
  };

  const int nk = K / BK;  // >= 2 (host)
#pragma unroll
  for (int j = 0; j < IPW; ++j) dma16_s(gbase(j, false), voff[j], sbase + j * 1024);
#pragma unroll
  for (int j = 0; j < IPW; ++j) dma16_s(gbase(j, false) + RB, voff[j], sbase + STAGE + j * 1024);
  // the next tile's offsets while stage 0 lands (needed from step nk - 2 on)
  int Ln = L + int(gridDim.x);
  if (Ln < total) {
    tn = tile(Ln);
    offsets(tn, vnx);
    bstep[0] = base_of(tn, K0) - bnow[0];
    bstep[1] = base_of(tn, K1) - bnow[1];
  }
  wait_vm<IPW>();
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NF; ++q) read_piece(0, 0, q);

  int ph = 0;  // buffer of the tile's stage 0
  for (;;) {
    const bool more = Ln < total;
    // one K step; in the tile's first (FIRST) the slice-0 products start the
    // accumulators
    auto kstep = [&](int kt, auto first) {
      constexpr bool FIRST = decltype(first)::value;
      const int buf = (kt + ph) & 1;
      // stage kt + 2: of this tile, else the next tile's stage kt + 2 - nk,
      // else (the block's last tile) this tile's last stage again, unused
      const bool nxt = kt + 2 >= nk && more;
      const int kn = kt + 2 < nk ? kt + 2 : more ? kt + 2 - nk : nk - 1;
      auto dma_slot = [&](int pos) {  // transfer pos / GAP at slot pos
        if (pos >= 0 && pos % GAP == 0 && pos / GAP < IPW) {
          const int j = pos / GAP;
          dma16_s(gbase(j, nxt) + kn * RB, nxt ? vnx[j] : voff[j], sbase + buf * STAGE + j * 1024);
        }
      };
      // slice 0: MFMAs on set 0, the reads of slice 1 into set 1 after the
      // first NF of them, the first barrier after MFMA B1J
#pragma unroll
      for (int j = 0; j < NM; ++j) {
        if constexpr (FIRST)
          mma_first(0, j);
        else
          mma(0, j);
        if (j < NF) read_piece(1, buf, j);
        if (j == B1J) __syncthreads();  // every wave's reads of stage kt are in
        if (j > B1J) dma_slot(j - B1J - 1);
      }
      // slice 1: MFMAs on set 1, the barrier, then the reads of stage
      // kt + 1, slice 0, into set 0 (unused in the last step: the registers
      // are free while the results are written, and read again after)
#pragma unroll
      for (int j = 0; j < NM; ++j) {
        if (j == RS) {
          // stage kt + 1 has landed: loads complete in issue order and only
          // stage kt + 2 may be out (stores in between do not matter)
          wait_vm<IPW>();
          __syncthreads();  // ... in every wave's part
        }
        mma(1, j);
        if (j < RS) dma_slot(NM - 1 - B1J + j);
        if (j >= RS && j - RS < NF) read_piece(0, buf ^ 1, j - RS);
      }
    };
    issue_scales(tc);
    kstep(0, std::true_type{});
    for (int kt = 1; kt < nk; ++kt) kstep(kt, std::false_type{});
    // the last MFMAs' results are read below: let them drain first
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int i = 0; i < MI; ++i) acc_fence_row<NI>(acc[i]);
    if constexpr (P::Op::INT)
      p.store_w4(tc, acc, (const float *)(smem + 2 * STAGE) + wave * NSC, wm, wn, pinned_lane());
    else
      p.store_w4(tc, acc, wm, wn, pinned_lane());
    if (!more) break;
    ph ^= nk & 1;
    // the next tile's stage 0 is in buffer ph (published by the last step's barrier)
#pragma unroll
    for (int q = 0; q < NF; ++q) read_piece(0, ph, q);
    L = Ln;
    tc = tn;
#pragma unroll
    for (int j = 0; j < IPW; ++j) voff[j] = vnx[j];
    bnow[0] += bstep[0];
    bnow[1] += bstep[1];
    Ln = L + int(gridDim.x);
    if (Ln < total) {
      tn = tile(Ln);
      offsets(tn, vnx);
      bstep[0] = base_of(tn, K0) - bnow[0];
      bstep[1] = base_of(tn, K1) - bnow[1];
    }
  }
}

// ------------------------------------------------------------------ launchers
// m_tiles bounds the row tiles (for grouped problems: the most any routing
// can need); the kernel takes the actual count from the problem.
template <class P, int BM, int BN, int WM, int WN, int BK, int S, int KW = 1>
inline hipError_t launch(const P &p, int K, int m_tiles, int n_tiles, hipStream_t st) {
  if (m_tiles > 0 && n_tiles > 0)
    gemm_mfma_kernel<P, BM, BN, WM, WN, BK, S, KW>
        <<<m_tiles * n_tiles, 64 * WM * WN * KW, 0, st>>>(p, K, n_tiles);
  return hipGetLastError();
}

// One block per CU at most (a block holds 128 KB of LDS), each walking its
// share of the tiles.
template <class P, int BM, int BN>
inline hipError_t launch_w4(const P &p, int K, int m_tiles, int n_tiles, hipStream_t st) {
  const int cu = cu_count();
  if (m_tiles > 0 && n_tiles > 0)
    gemm_w4_kernel<P, BM, BN><<<std::min(m_tiles * n_tiles, cu), 256, 0, st>>>(p, K, n_tiles);
  return hipGetLastError();
}

// The four-wave kernel addresses operand rows by 32-bit byte offsets from the
// lowest of an operand's matrices: *lo gets that pointer, and the result says
// whether every matrix ends within 4 GB of it.
struct Span {
  const void *p;
  size_t bytes;
};
template <class E>
inline bool span32(std::initializer_list<Span> ms, const E **lo) {
  uintptr_t a = UINTPTR_MAX, b = 0;
  for (const Span &m : ms) {
    a = std::min(a, uintptr_t(m.p));
    b = std::max(b, uintptr_t(m.p) + m.bytes);
  }
  *lo = (const E *)a;
  return b - a < (uintptr_t(1) << 32);
}

// Choice of the tile of a product of N rows and c128 columns of 128.  A tile
// shape costs its rounds over the CUs (slots of a round: blocks resident at
// once) times the time of one round, relative to the 128 x 128 tile's with
// two blocks of four waves a CU (40 us at K 2048, 22 us at K 1024):
//   128 x 128, eight waves, three stages, one block a CU  0.65, one round only
//   64 x 128, two stages, three blocks a CU               0.9
//   256 x 128 / 192 / 256, four waves, one block a CU     0.95 / 1.15 / 1.3
// The large tiles win where they fill their rounds, the small ones in
// between.  Measured (us; weights not in a cache; before: the 32-row tiles up
// to 2048 tokens and the four-wave kernel above): 1.3B QKV 700 tokens 39 -> 26,
// 1000 44 -> 27, 2000 87 -> 42, 2500 56 -> 44; 410M QKV 2500 22 -> 18, 6000
// 41 -> 34; 160M QKV 8192 36 -> 29; 1.3B O-projection 2000 57 -> 24, 4096 50 -> 40;
// 410M 2500 25 -> 13, 4096 27 -> 14; 160M 4096 18 -> 11; the full batches
// (16384) keep the four-wave tiles, but for 160M QKV (51 -> 48).
constexpr float COST_ONE_ROUND = 0.65f, COST_64X128 = 0.9f, COST_128X128 = 1.f,
                COST_256X128 = 0.95f, COST_256X192 = 1.15f, COST_256X256 = 1.3f;
inline float tile_cost(int tiles, float cost, int per_cu = 1) {
  const int slots = cu_count() * per_cu;
  return float((tiles + slots - 1) / slots) * cost;
}
inline int tiles64(int N, int c128) { return (N + 63) / 64 * c128; }
inline int tiles128(int N, int c128) { return (N + 127) / 128 * c128; }
inline bool one_round(int t128) { return t128 <= cu_count(); }
// the four-wave kernel's rounds, at cost t, beat the smaller tiles'
inline bool w4_rounds(int N, int c128, float t) {
  if (one_round(tiles128(N, c128))) return t <= COST_ONE_ROUND;
  return t <= std::min(tile_cost(tiles64(N, c128), COST_64X128, 3),
                       tile_cost(tiles128(N, c128), COST_128X128, 2));
}
// Below 192 tiles of 64 x 128 most CUs would have none: the 32-row tiles
// stream the weights from more of them (410M QKV 512 tokens, 96 tiles: 12.4
// against 13.9 us; 1.3B QKV 512 tokens, 192 tiles: 29.5 against 23.5 us).
inline bool few_tiles(int N, int c128) { return tiles64(N, c128) < 192; }

// At most one 32 x 64 block a CU: two K groups in the block (1.3B O-projection,
// 1 to 128 tokens, 32 to 128 blocks: 12.4 to 13.0 -> 8.7 to 10.1 us; at 352
// blocks 15.0 -> 19.4 us).
inline bool split_k(int blocks, int K) { return blocks <= cu_count() && K % 128 == 0; }

// Up to 288 tiles of 64 rows, three stages: the blocks wait on each step's
// transfers (1.3B O-projection, 1000 tokens, 256 tiles: 19.2 us, with two
// stages 29.3, the 128-row tiles 22.2).
template <class P>
inline hipError_t launch_mid(const P &p, int K, int N, int c128, hipStream_t st) {
  const int m64 = (N + 63) / 64, m128 = (N + 127) / 128;
  if (tiles64(N, c128) <= 288) return launch<P, 64, 128, 2, 2, 64, 3>(p, K, m64, c128, st);
  if (one_round(m128 * c128)) return launch<P, 128, 128, 4, 2, 64, 3>(p, K, m128, c128, st);
  if (tile_cost(m64 * c128, COST_64X128, 3) <= tile_cost(m128 * c128, COST_128X128, 2))
    return launch<P, 64, 128, 2, 2, 64, 2>(p, K, m64, c128, st);
  return launch<P, 128, 128, 2, 2, 64, 2>(p, K, m128, c128, st);
}
}  // namespace tr
