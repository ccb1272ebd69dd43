// Tiles of 32 rows in LDS as the fp32 matrix kernels hold them: staging, operand reads and the two products
// (layout: s2attn_f32.hip).
#pragma once
#include "s2attn_f32_common.h"

namespace s2 {
namespace {

constexpr int kTile = 32;     // rows of a staged tile
constexpr int kWgRows = 64;   // rows a workgroup owns: 16 per wave

template <int D>
struct Lanes {
  static constexpr int kRow = D * 4;             // bytes of a tile row
  static constexpr int kTileBytes = kTile * kRow;
  int rm[2];   // row-major operand: byte offset for even / odd i, + 128 (i / 2)
  int tr[4];   // transposed operand of register v, + 256 j
  int st_row;  // staging: tile row of this lane's first 16 bytes, and its chunk
  int st_chunk;

  __device__ __forceinline__ void init(int lane, int w) {
    const int c16 = lane & 15, q4 = lane >> 4;
    rm[0] = c16 * kRow + ((q4 ^ (c16 & 7)) << 4);
    rm[1] = c16 * kRow + (((4 + q4) ^ (c16 & 7)) << 4);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int row = 4 * q4 + v;
      tr[v] = row * kRow + ((c16 ^ (row & 7)) << 4);
    }
    constexpr int kChunks = D / 4;               // 16-byte chunks of a row: 16 or 32
    constexpr int kRowsPer = 64 / kChunks;       // rows one wave instruction fills: 4 or 2
    st_row = w * kRowsPer + lane / kChunks;
    st_chunk = (lane % kChunks) ^ (st_row & 7);
  }

  // X[16 RB + c16][16 i + 4 q4 ..]
  template <int RB>
  __device__ __forceinline__ f32x4 row(const char* tile, int i) const {
    return *reinterpret_cast<const f32x4*>(tile + rm[i & 1] + 16 * RB * kRow + 128 * (i >> 1));
  }
  // X[16 RB + 4 q4 + v][64 j + 4 c16 ..]
  template <int RB>
  __device__ __forceinline__ f32x4 col(const char* tile, int v, int j) const {
    return *reinterpret_cast<const f32x4*>(tile + tr[v] + 16 * RB * kRow + 256 * j);
  }

  // Stages rows i0 .. i0 + 31 of a run (clamped to its last row) of one head.
  __device__ __forceinline__ void stage(const KArgs& a, const Run& run, int s, const void* src, const TStride& st,
                                        int b, int head, int i0, uint32_t lds, int w) const {
    constexpr int kStep = 4 * (64 / (D / 4));    // rows the four waves fill together: 16 or 8
#pragma unroll
    for (int p = 0; p < kTile / kStep; ++p) {
      const int tok = run_token(a, run, i0 + p * kStep + st_row, s);
      dma16(static_cast<const char*>(src) + row_off(st, b, tok, head) * 4 + (st_chunk << 4), lds + (p * 4 + w) * 1024);
    }
  }
};

// acc[RB] += rows of the tile (16 RB + c16) against the wave's own 16 rows held in `own`.
template <int D>
__device__ __forceinline__ void scores(f32x4 (&acc)[2], const char* tile, const Lanes<D>& ln, const f32x4 (&own)[D / 16]) {
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const f32x4 x0 = ln.template row<0>(tile, i), x1 = ln.template row<1>(tile, i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[0] = mfma4(x0[e], own[i][e], acc[0]);
      acc[1] = mfma4(x1[e], own[i][e], acc[1]);
    }
  }
}

// acc[j][e] += X^T W for the 32 rows of a tile: W = P or dS as it stands in the accumulators.
template <int D>
__device__ __forceinline__ void accumulate(f32x4 (&acc)[D / 64][4], const char* tile, const Lanes<D>& ln, const f32x4 (&wt)[2]) {
#pragma unroll
  for (int v = 0; v < 4; ++v)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const f32x4 x0 = ln.template col<0>(tile, v, j), x1 = ln.template col<1>(tile, v, j);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = mfma4(x0[e], wt[0][v], acc[j][e]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = mfma4(x1[e], wt[1][v], acc[j][e]);
    }
}

}  // namespace
}  // namespace s2
