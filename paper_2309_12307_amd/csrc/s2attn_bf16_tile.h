// The two tile layouts of the bf16 kernels (head dimension 128 and 64) under one name, for kernels that take the head
// dimension as a template parameter.
#pragma once
#include "s2attn_bf16_common.h"
#include "s2attn_bf16_tile64.h"

namespace s2 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Sixteen e4m3 values times 2^(exps - 127) as bf16: exact, the products have four significant bits.
template <class Vec>
__device__ __forceinline__ void widen(const Vec& u, float scale, bf16x8& lo, bf16x8& hi) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  bf16x2 p[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
    p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[2 * i] = p[i][0]; lo[2 * i + 1] = p[i][1];
    hi[2 * i] = p[4 + i][0]; hi[2 * i + 1] = p[4 + i][1];
  }
}

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
