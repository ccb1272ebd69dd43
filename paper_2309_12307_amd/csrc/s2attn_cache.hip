// Writing new tokens' K and V into the paged cache, and reading cached rows back.  Both only move memory: what bounds
// them is HBM (write: 2 T Hkv D elements in, as many out; read: the reverse).  32 heads, D = 128, bf16 rows, e4m3 cache: 32768 tokens
// written 148 us (5.4 TB/s), 100 000 read back 522 us (4.7 TB/s; a copy of 4 GB 4.8).  Single tokens are latency: 3.9 us.
//
// An e4m3 cache holds of every row (token, kv head) of D values x the values rn(x 2^-e) and the exponent e, the least
// with max |x| <= 448 * 2^e.  The scale is a power of two because the values are floating: their relative step is the same
// under any scale, so a finer one would buy nothing, and with this one neither scaling nor reading back (also to bf16) rounds.
// Infinities and NaN are stored as NaN and have no part in the maximum.
//
// A lane moves 16 bytes of a cached row (4, 8 or 16 values), the rows of K and then of V of one token after the other.  A wave
// has up to kSteps such pieces a lane, of one token or, where one has too few for 64 lanes, of several; its loads of the call's
// rows go out before it looks for the token's place (three dependent reads).  Consecutive tokens stay on one XCD, so that its
// L2 gathers the exponents, a byte a row, to whole lines.
#include "s2attn_bf16_tile.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

enum { kBf16 = 0, kF32 = 1, kE4m3 = 2 };
constexpr int kBytes[3] = {2, 4, 1};
constexpr int kSteps = 4;   // pieces of a lane, in flight together

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// A lane's values as the call's rows hold them.
template <int ROWS, int V>
struct Values {
  static constexpr int N = V * kBytes[ROWS] / 16;
  u32x4 x[N];
  __device__ __forceinline__ uint32_t word(int i) const {
    return x[i >> 2][i & 3];
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (ROWS == kBf16) return __uint_as_float(i & 1 ? word(i >> 1) & 0xffff0000u : word(i >> 1) << 16);
    else return __uint_as_float(word(i));
  }
};

template <int X>
__device__ __forceinline__ uint32_t max_dpp(uint32_t u) {
  return max(u, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, X, 0xf, 0xf, true));
}
// Maximum over 4 or 8 neighbouring lanes: quad_perm [1,0,3,2] and [2,3,0,1], row_half_mirror.
template <int LANES>
__device__ __forceinline__ uint32_t max_lanes(uint32_t u) {
  static_assert(LANES == 4 || LANES == 8, "lanes of a row");
  u = max_dpp<0x4E>(max_dpp<0xB1>(u));
  return LANES == 8 ? max_dpp<0x141>(u) : u;
}

// Biased exponent of a row whose largest finite |x| has these bits.  amax = m 2^x: e = x - 8, and one more where m is
// over 1.75 = 448 / 256.
__device__ __forceinline__ int exponent_of(uint32_t top) {
  return min(max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 17), 247);
}

// A row's values as e4m3 (LANES lanes of 16), and its biased exponent.  By the bits: this build's floating-point flags know no
// NaN.
template <int ROWS, int LANES>
__device__ __forceinline__ u32x4 quantise(const Values<ROWS, 16>& x, int& e) {
  uint32_t top = 0;
  if constexpr (ROWS == kBf16) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x.word(i) & 0x7fff7fffu));
    top = (uint32_t)max(m[0], m[1]) << 16;
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, x.word(i) & 0x7fffffffu);
  }
  top = max_lanes<LANES>(top);
  s16x2 out[4];
  if (__builtin_amdgcn_ballot_w64(top >= 0x7f800000u) == 0) {
    e = exponent_of(top);
    const float scale = __uint_as_float((uint32_t)e << 23);   // the conversion divides by it
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s16x2 u = {0, 0};
      if constexpr (ROWS == kBf16) {
        u = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(u, __builtin_bit_cast(bf16x2, x.word(2 * i)), scale, false);
        u = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(u, __builtin_bit_cast(bf16x2, x.word(2 * i + 1)), scale, true);
      } else {
        u = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(u, x.value(4 * i), x.value(4 * i + 1), scale, false);
        u = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(u, x.value(4 * i + 2), x.value(4 * i + 3), scale, true);
      }
      out[i] = u;
    }
    return u32x4{__builtin_bit_cast(uint32_t, out[0]), __builtin_bit_cast(uint32_t, out[1]),
                 __builtin_bit_cast(uint32_t, out[2]), __builtin_bit_cast(uint32_t, out[3])};
  }
  // some row of the wave holds an infinity or a NaN: they leave the maximum alone and become NaN
  top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t u = __float_as_uint(x.value(i)) & 0x7fffffffu;
    top = max(top, u < 0x7f800000u ? u : 0u);
  }
  e = exponent_of(max_lanes<LANES>(top));
  const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f[4];
    uint32_t nan = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t u = __float_as_uint(x.value(4 * i + k));
      const bool off = (u & 0x7fffffffu) >= 0x7f800000u;
      f[k] = off ? 0.f : __uint_as_float(u) * inv;
      nan |= off ? (0x7fu | (u >> 24 & 0x80u)) << (8 * k) : 0u;
    }
    uint32_t v = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    r[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], v, true) | nan;
  }
  return u32x4{r[0], r[1], r[2], r[3]};
}

// Sixteen e4m3 values times 2^(exponent - 127).
template <int ROWS>
__device__ __forceinline__ Values<ROWS, 16> restore(const u32x4& u, float scale) {
  Values<ROWS, 16> r;
  if constexpr (ROWS == kBf16) {
    bf16x8 lo, hi;
    widen(u, scale, lo, hi);
    r.x[0] = __builtin_bit_cast(u32x4, lo);
    r.x[1] = __builtin_bit_cast(u32x4, hi);
  } else {
    const uint32_t w[4] = {u[0], u[1], u[2], u[3]};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
      r.x[i] = __builtin_bit_cast(u32x4, f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale});
    }
  }
  return r;
}

template <int D, int ROWS, int CACHE, bool WRITE>
__global__ void __launch_bounds__(256) cache_kernel(PArgs a, int tokens, Div by_waves, int blocks, int first_block) {
  constexpr int V = 16 / kBytes[CACHE], kLanes = D / V;
  using X = Values<ROWS, V>;
  const int lane = thread_id() & 63, id = first_block + block_id();
  const int block = (id & 7) * (blocks >> 3) + (id >> 3);   // consecutive blocks on one XCD
  const int wave = uni(block * 4 + (thread_id() >> 6));
  const int unit = quot(wave, by_waves);                    // `tokens` tokens
  const int items = 2 * a.Hkv * kLanes;                     // pieces of a token
  const int waves = (items * tokens + 64 * kSteps - 1) / (64 * kSteps);
  const int part = wave - unit * waves;
  const int t0 = unit * tokens;
  if (t0 >= a.T) return;

  int t[kSteps], c[kSteps], chunk[kSteps];
  bool is_v[kSteps], on[kSteps];
  u32x4 x[kSteps][X::N];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    int i = (part * kSteps + s) * 64 + lane;
    on[s] = i < items * tokens;
    t[s] = t0;
    if (tokens > 1) {                                       // items is then a power of two
      t[s] += i / items;
      i &= items - 1;
    }
    on[s] = on[s] && t[s] < a.T;
    const int row = i / kLanes;
    chunk[s] = i % kLanes;
    is_v[s] = row >= a.Hkv;
    c[s] = is_v[s] ? row - a.Hkv : row;
    if constexpr (WRITE) {
      const long long off = on[s] ? (is_v[s] ? t[s] * a.v_t + c[s] * a.v_h : t[s] * a.k_t + c[s] * a.k_h) + chunk[s] * V : 0;
      const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const char*>(is_v[s] ? a.v : a.k) + off * kBytes[ROWS]);
#pragma unroll
      for (int n = 0; n < X::N; ++n) x[s][n] = src[n];
    }
  }

  // the places of the tokens: their sequences' positions, and whether they are rows of one
  int b[kSteps], pos[kSteps], keys[kSteps];
  bool mine[kSteps];
  CacheRow at[kSteps];
  if (tokens == 1) {
    const SeqRows sr = find_rows<-1>(a, t0, lane);
    const bool in = sr.b >= 0 && t0 >= sr.s0 && t0 < sr.s0 + sr.n;
    const int p = sr.kv - sr.n + (t0 - sr.s0);
    const CacheRow one = cache_row(a, sr.b, p, in && p >= 0 && p < sr.keys);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) { at[s] = one; mine[s] = in; }
  } else {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) { b[s] = 0; pos[s] = -1; keys[s] = 0; mine[s] = false; }
    for (int u = 0; u < tokens && t0 + u < a.T; ++u) {
      const SeqRows sr = find_rows<-1>(a, t0 + u, lane);
      const bool in = sr.b >= 0 && t0 + u >= sr.s0 && t0 + u < sr.s0 + sr.n;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        if (in && t[s] == t0 + u) { b[s] = sr.b; pos[s] = sr.kv - sr.n + (t0 + u - sr.s0); keys[s] = sr.keys; mine[s] = true; }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) at[s] = cache_row(a, b[s], pos[s], pos[s] >= 0 && pos[s] < keys[s]);
  }
  u32x4 y[kSteps];
  float scale[kSteps];
  u32x4* cached[kSteps];
  uint8_t* exps[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const bool there = on[s] && at[s].page >= 0;
    const long long cp = is_v[s] ? a.vc_p : a.kc_p, ct = is_v[s] ? a.vc_t : a.kc_t, ch = is_v[s] ? a.vc_h : a.kc_h;
    cached[s] = reinterpret_cast<u32x4*>((is_v[s] ? a.vc : a.kc) + (at[s].page * cp + at[s].at * ct + c[s] * ch + chunk[s] * V) * kBytes[CACHE]);
    if constexpr (CACHE == kE4m3)
      exps[s] = is_v[s] ? a.ve + at[s].page * a.ve_p + at[s].at * a.ve_t + c[s] * a.ve_h
                        : a.ke + at[s].page * a.ke_p + at[s].at * a.ke_t + c[s] * a.ke_h;
    if constexpr (!WRITE) {
      y[s] = u32x4{0, 0, 0, 0};                             // no such position, or no page: zeros
      scale[s] = 1.f;
      if (there) {
        y[s] = *cached[s];
        if constexpr (CACHE == kE4m3) scale[s] = __uint_as_float((uint32_t)*exps[s] << 23);
      }
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const bool there = on[s] && at[s].page >= 0;
    if constexpr (WRITE) {
      if constexpr (CACHE == kE4m3) {
        int e;
        X row;
#pragma unroll
        for (int n = 0; n < X::N; ++n) row.x[n] = x[s][n];
        const u32x4 q = quantise<ROWS, kLanes>(row, e);     // all lanes of a row are here together
        if (there) {
          *cached[s] = q;
          if (chunk[s] == 0) *exps[s] = (uint8_t)e;
        }
      } else if (there) {
        *cached[s] = x[s][0];
      }
    } else if (on[s] && mine[s]) {
      const long long off = (is_v[s] ? t[s] * a.v_t + c[s] * a.v_h : t[s] * a.k_t + c[s] * a.k_h) + chunk[s] * V;
      u32x4* dst = reinterpret_cast<u32x4*>(static_cast<char*>(is_v[s] ? a.v : a.k) + off * kBytes[ROWS]);
      if constexpr (CACHE == kE4m3) {
        const auto r = restore<ROWS>(y[s], scale[s]);
#pragma unroll
        for (int n = 0; n < r.N; ++n) dst[n] = r.x[n];
      } else {
        *dst = y[s];
      }
    }
  }
}

template <int D, int ROWS, int CACHE, bool WRITE>
int launch(const PArgs& a, hipStream_t st) {
  const int items = 2 * a.Hkv * (D * kBytes[CACHE] / 16);
  const int tokens = items < 64 && (items & (items - 1)) == 0 ? 64 / items : 1;
  const int waves = (items * tokens + 64 * kSteps - 1) / (64 * kSteps);
  const long long total = (long long)((a.T + tokens - 1) / tokens) * waves;
  const int blocks = (int)((total + 31) / 32) * 8;
  return launch_blocks(cache_kernel<D, ROWS, CACHE, WRITE>, blocks, 256, st, a, tokens, div_by(waves), blocks);
}

template <int D, bool WRITE>
int launch_types(const PArgs& a, int dtype, int cache, hipStream_t st) {
  if (dtype == kBf16) return cache == kE4m3 ? launch<D, kBf16, kE4m3, WRITE>(a, st) : launch<D, kBf16, kBf16, WRITE>(a, st);
  return cache == kE4m3 ? launch<D, kF32, kE4m3, WRITE>(a, st) : launch<D, kF32, kF32, WRITE>(a, st);
}

}  // namespace

int launch_cache_write(const PArgs& a, int D, int dtype, int cache, hipStream_t st) {
  return D == 64 ? launch_types<64, true>(a, dtype, cache, st) : launch_types<128, true>(a, dtype, cache, st);
}
int launch_cache_read(const PArgs& a, int D, int dtype, int cache, hipStream_t st) {
  return D == 64 ? launch_types<64, false>(a, dtype, cache, st) : launch_types<128, false>(a, dtype, cache, st);
}

}  // namespace s2
