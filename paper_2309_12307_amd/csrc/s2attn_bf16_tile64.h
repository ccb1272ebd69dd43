// LDS tile layout of the bf16 kernels for head dimension 64: rows of 128 bytes, and the operand fragments read from them
// (operand layouts of the matrix instruction: s2attn_bf16_common.h).
#pragma once
#include "s2attn_bf16_common.h"

namespace s2 {

constexpr int kRow64 = 64 * 2;          // bytes of a tile row

// Tile rows 2R and 2R + 1 share the 256-byte LDS row R; its eight chunk columns are XOR-permuted
// by a function of R mod 8 that takes every value (16 rows of one chunk column hit all banks) and
// differs in bit 2 between neighbouring R (4 rows x 64 bytes of a transposing read do too).
__device__ __forceinline__ int swz64(int R) { return ((R & 1) << 2) | ((R >> 1) & 3); }
__device__ __forceinline__ int tile_off64(int row, int chunk) {
  return (row >> 1) * 256 + ((row & 1) << 7) + ((chunk ^ swz64(row >> 1)) << 4);
}

struct Offsets64 {
  int rm[4];      // row-major fragment k: elements [16k + 8g, +8) of row l % 32
  int tr[2][2];   // transposed fragment, column block cb: rows 4g + L/4 and that + 8
};
__device__ __forceinline__ Offsets64 lane_offsets64(int lane) {
  Offsets64 o;
  const int l32 = lane & 31, g32 = lane >> 5, L = lane & 15;
#pragma unroll
  for (int k = 0; k < 4; ++k) o.rm[k] = tile_off64(l32, 2 * k + g32);
  const int row = 4 * g32 + (L >> 2);
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const int col = 32 * cb + (lane & 16) + 4 * (L & 3);
    o.tr[cb][0] = tile_off64(row, col >> 3) + (col & 7) * 2;
    o.tr[cb][1] = tile_off64(row + 8, col >> 3) + (col & 7) * 2;
  }
  return o;
}
template <int ROW0>   // a multiple of 16
__device__ __forceinline__ bf16x8 rm64(const char* tile, const Offsets64& o, int k) {
  return *reinterpret_cast<const bf16x8*>(tile + o.rm[k] + ROW0 * kRow64);
}
template <int ROW0>
__device__ __forceinline__ bf16x8 tr64(const char* tile, const Offsets64& o, int cb) {
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(S2_LDS(bf16x4, tile + o.tr[cb][0] + ROW0 * kRow64));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(S2_LDS(bf16x4, tile + o.tr[cb][1] + ROW0 * kRow64));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

}  // namespace s2
