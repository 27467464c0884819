// Pieces that the bf16 MFMA products share (gfx950): operand types, the order in
// which tiles are handed to the XCDs, the LDS swizzle of K-contiguous stages and
// products on the accumulator registers.
#pragma once

#include "common.hpp"

namespace tr {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Tiles of the whole problem are handed out XCD by XCD: blocks are issued to
// the 8 XCDs round-robin, so block L runs on XCD L % 8, and it takes tile
// number (its XCD's contiguous share) + L / 8.  Tile t covers row tile t / ny
// and column tile t % ny, so the blocks resident on one XCD share A rows and
// a few weight tiles in that XCD's L2.
__device__ __forceinline__ int xcd_tile(int L, int total) {
  const int per = total >> 3, extra = total & 7, x = L & 7;
  return x * per + min(x, extra) + (L >> 3);
}

// Order of the tiles handed to one XCD.  The 32 CUs of an XCD run 32
// consecutive tiles of its share at a time and stream their K loops in near
// lockstep, so what that XCD's L2 must hold per K step is the union of their
// operand slices.  Walking the tiles in bands of BAND_R row tiles (of one
// expert, for grouped problems), each band in chunks of BAND_R x BAND_C
// tiles with the row fastest, makes that union BAND_R A slices and BAND_C B
// slices instead of one A slice and 32 B slices (the expert weights would
// otherwise stream past the L2 once per row tile).
constexpr int BAND_R = 16, BAND_C = 2;

// Tile t of a rows x ny grid walked in bands -> (row tile i, column tile j).
template <int BR = BAND_R, int BC = BAND_C>
__device__ __forceinline__ void band_order(int t, int rows, int ny, int &i, int &j) {
  const int band = t / (BR * ny);
  const int rem = t - band * BR * ny;
  const int rb = min(BR, rows - band * BR);  // rows of this band
  const int chunk = rem / (rb * BC);
  const int idx = rem - chunk * rb * BC;
  i = band * BR + idx % rb;
  j = chunk * BC + idx / rb;
}

// LDS chunk (16 bytes) of chunk c of operand row r in a stage whose rows are
// CPR chunks long: a XOR with the row's position in its 256-byte bank span
// makes the 16 rows read by one 16-lane phase (same c) hit 16 distinct
// 16-byte bank groups.
template <int CPR>
__device__ __forceinline__ int swz(int r, int c) {
  if constexpr (CPR == 8)
    return c ^ ((r >> 1) & 7);  // 2 rows per 256-byte span
  else
    return c ^ ((r >> 2) & 3);  // 4 rows per span
}

// vmcnt(n * N) for the run-time n of stages still allowed in flight, n < S - 1
template <int N, int S>
__device__ __forceinline__ void wait_stages(int n) {
  if constexpr (S > 5) if (n >= 4) { wait_vm<4 * N>(); return; }
  if constexpr (S > 4) if (n == 3) { wait_vm<3 * N>(); return; }
  if constexpr (S > 3) if (n == 2) { wait_vm<2 * N>(); return; }
  if constexpr (S > 2) if (n == 1) { wait_vm<N>(); return; }
  wait_vm<0>();
}

// acc += a b on the accumulator registers (AGPRs).  With 256 accumulators
// per lane the register allocator, left to itself, parks some of them in
// VGPRs and copies them around every MFMA; pinning them to AGPRs keeps the
// loop free of copies.  As a volatile asm statement it also keeps its place
// relative to the LDS reads and transfers written around it, so the program
// order below is the issue order.
__device__ __forceinline__ void mfma_agpr(f32x4_t &acc, const bf16x8_t &a, const bf16x8_t &b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// acc = a b (the first product of a tile: no zeroing of the accumulators)
__device__ __forceinline__ void mfma_agpr_first(f32x4_t &acc, const bf16x8_t &a, const bf16x8_t &b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=a"(acc) : "v"(a), "v"(b));
}

// The compiler does not see the MFMAs inside the asm statements, so it does
// not keep its own accesses of the accumulators clear of their hazards.
// Each row of accumulators passes through an asm statement that starts with
// `nops` wait states: accesses after it are ordered after the wait, and
// writes before it (zeroing) before the wait.
template <int NI>
__device__ __forceinline__ void acc_fence_row(f32x4_t (&a)[NI]) {
  static_assert(NI == 4 || NI == 6 || NI == 8, "accumulator row widths in use");
  if constexpr (NI == 4)
    asm volatile("s_nop 4" : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]));
  else if constexpr (NI == 8)
    asm volatile("s_nop 4" : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]), "+a"(a[4]), "+a"(a[5]),
                 "+a"(a[6]), "+a"(a[7]));
  else
    asm volatile("s_nop 4" : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]), "+a"(a[4]), "+a"(a[5]));
}

}  // namespace tr
