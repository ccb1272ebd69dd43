// The two tile layouts of the bf16 kernels (head dimension 128 and 64) under one name, for kernels that take the head
// dimension as a template parameter.
#pragma once
#include "s2attn_bf16_common.h"
#include "s2attn_bf16_tile64.h"

namespace s2 {

template <int D>
struct Tile;
template <>
struct Tile<128> {
  static constexpr int kRow = kRowBytes;
  LaneOffsets o;
  __device__ __forceinline__ void init(int lane) { init_lane_offsets(o, lane); }
  static __device__ __forceinline__ int off(int row, int chunk) { return tile_off(row, chunk); }
  template <int ROW0>
  __device__ __forceinline__ bf16x8 rm(const char* tile, int k) const { return frag_rm<ROW0>(tile, o, k); }
  template <int ROW0>
  __device__ __forceinline__ bf16x8 tr(const char* tile, int cb) const { return frag_tr<ROW0>(tile, o, cb); }
};
template <>
struct Tile<64> {
  static constexpr int kRow = kRow64;
  Offsets64 o;
  __device__ __forceinline__ void init(int lane) { o = lane_offsets64(lane); }
  static __device__ __forceinline__ int off(int row, int chunk) { return tile_off64(row, chunk); }
  template <int ROW0>
  __device__ __forceinline__ bf16x8 rm(const char* tile, int k) const { return rm64<ROW0>(tile, o, k); }
  template <int ROW0>
  __device__ __forceinline__ bf16x8 tr(const char* tile, int cb) const { return tr64<ROW0>(tile, o, cb); }
};

}  // namespace s2
