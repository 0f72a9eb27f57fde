// Pieces shared by the bf16 matrix product kernels (the transformer block's and the affine
// map's): swizzled LDS tiles, their fragments, and barriers that leave loads in flight.
#pragma once
#include "common.hpp"

namespace bsa {
namespace {

// 16-byte chunk swizzle of a staged tile row: 4 or 8 chunks per row (row-fragment reads
// of 16 consecutive rows on distinct banks) or 16 and more chunks per row (transposing
// reads of 8 consecutive rows, chunk pairs on distinct banks).
// MIX: transposing reads of rows 8j + {0..3} (+ 4) instead, for a tile whose partner is read in
// row fragments (rows 0-3 and 8-11, 4-7 and 12-15, .. on distinct banks).
template <int COLS, bool MIX = false>
__device__ __forceinline__ int tile_swz(int x) {
  if (MIX) return COLS == 64 ? 2 * (((x >> 1) & 1) | ((x >> 2) & 2)) : 2 * ((x & 3) | ((x >> 1) & 4));
  return COLS == 32 ? ((x >> 1) & 3) : COLS == 64 ? (x & 7) : 2 * (x & 7);
}

template <int BK>
__device__ __forceinline__ bf16x8 frag_row(const bf16_t* t, int row, int lc) {
  return *reinterpret_cast<const bf16x8*>(t + row * BK + 8 * (lc ^ tile_swz<BK>(row)));
}

// Workgroup barrier without a memory fence: the waves' direct-to-LDS loads are already
// waited for by each wave (vmcnt), and later tiles stay in flight across it (the fence of
// __syncthreads would wait for every outstanding load). The empty statements keep the
// compiler from moving LDS accesses across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// s_waitcnt with vmcnt = V (expcnt and lgkmcnt left at their maxima)
template <int V>
__device__ __forceinline__ void vm_wait() {
  static_assert(V >= 0 && V < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((V & 15) | ((V >> 4) << 14) | (7 << 4) | (15 << 8));
}

// Wait for this wave's LDS reads; no LDS access moves across it.
__device__ __forceinline__ void lgkm_drain() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// LDS byte addresses of the two transposing reads that give lane (p = L % 16, j = L / 16)
// the operand X[k0 + 4j + i][m0 + p] (i = 0..3) and X[k0 + 16 + 4j + i][m0 + p] of a
// [BK][COLS] tile X (BK = 32 or 64): within each 16-lane group, ds_read_b64_tr_b16 hands lane l element
// l % 4 of the 4-element runs addressed by lanes l / 4, 4 + l / 4, 8 + l / 4, 12 + l / 4, so
// lane p addresses row k0 + 4j + p / 4 (then + 16) at columns m0 + 4 (p % 4) + [0, 4).
// MIX: X[k0 + 8j + i][m0 + p] and X[k0 + 8j + 4 + i][m0 + p] instead, the order of a row fragment.
template <int COLS, bool MIX>
__device__ __forceinline__ void tr_addr(const bf16_t* t, int k0, int m0, int lane, uint32_t& o0, uint32_t& o1) {
  const int p = lane & 15, j = lane >> 4;
  const int col = m0 + 4 * (p & 3);
  const int lc = col >> 3, sub = col & 7;
  const int x0 = k0 + (MIX ? 8 : 4) * j + (p >> 2), x1 = x0 + (MIX ? 4 : 16);
  const bf16_t* a0 = t + x0 * COLS + 8 * (lc ^ tile_swz<COLS, MIX>(x0)) + sub;
  const bf16_t* a1 = t + x1 * COLS + 8 * (lc ^ tile_swz<COLS, MIX>(x1)) + sub;
  o0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)a0;
  o1 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)a1;
}

// Four operand fragments (columns m0 + 16 i, i = 0..3) of one 32-deep contraction step of
// the transposed form, issued as one statement that also waits for them: every use of the
// results follows the wait.
template <int COLS, bool MIX = false>
__device__ __forceinline__ void tr_frags4(const bf16_t* t, int k0, int m0, int lane, bf16x8 (&f)[4]) {
  uint32_t a[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) tr_addr<COLS, MIX>(t, k0, m0 + 16 * i, lane, a[2 * i], a[2 * i + 1]);
  uint2 r[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9\n\t"
      "ds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %3, %11\n\t"
      "ds_read_b64_tr_b16 %4, %12\n\tds_read_b64_tr_b16 %5, %13\n\t"
      "ds_read_b64_tr_b16 %6, %14\n\tds_read_b64_tr_b16 %7, %15\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7])
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f[i] = __builtin_bit_cast(bf16x8, make_uint4(r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y));
}

// The same for two fragments (columns m0 and m0 + 16).
template <int COLS, bool MIX = false>
__device__ __forceinline__ void tr_frags2(const bf16_t* t, int k0, int m0, int lane, bf16x8 (&f)[2]) {
  uint32_t a[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) tr_addr<COLS, MIX>(t, k0, m0 + 16 * i, lane, a[2 * i], a[2 * i + 1]);
  uint2 r[4];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\t"
      "ds_read_b64_tr_b16 %2, %6\n\tds_read_b64_tr_b16 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3])
      : "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i)
    f[i] = __builtin_bit_cast(bf16x8, make_uint4(r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y));
}

// 1 / (1 + exp(-x)): the hardware reciprocal and one Newton step (within an ulp of the divided
// value, at a third of the division's instructions). Where exp(-x) leaves the range in which the
// reciprocal is a normal number (x below -87) the reciprocal stands: the step would give NaN.
__device__ __forceinline__ float sigmoid(float x) {
  const float y = 1.0f + __expf(-x);
  const float r = __builtin_amdgcn_rcpf(y);
  return y < 0x1p126f ? fmaf(fmaf(-y, r, 1.0f), r, r) : r;
}

// Rows of a wave's tile that pass through LDS at a time in the epilogue: as many as fit the
// four arrays of the first two stages.
constexpr int epi_rows(int array_bytes, int tmw, int tnw, int nw) {
  int rp = tmw;
  while (rp > 16 && 4 * (array_bytes / (rp * tnw * 4)) < nw) rp /= 2;
  return rp;
}

}  // namespace
}  // namespace bsa
