// Writing new tokens' K and V into the paged cache, and reading cached rows back.  Both only move memory: what bounds
// them is HBM (write: 2 T Hkv D elements in, as many out; read: the reverse).
//
// An e4m3 cache holds of every row (token, kv head) of D values x the values rn(x 2^-e) and the exponent e, the least
// with max |x| <= 448 * 2^e.  The scale is a power of two because the values are floating: their relative step is the same
// under any scale, so a finer one would buy nothing, and with this one neither scaling nor reading back (also to bf16) rounds.
// Infinities and NaN are stored as NaN and have no part in the maximum.
//
// A lane moves 8 values, D / 8 lanes a row, the rows of K and then of V of one token after the other; a wave takes the
// tokens of `tokens` rows of the call where one token has too few values for 64 lanes.  Its loads of the call's rows go out
// before it looks for the token's place (three dependent reads).
#include "s2attn_bf16_common.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

enum { kBf16 = 0, kF32 = 1, kE4m3 = 2 };

// Eight values as they are held: in registers as fp32 bits.
struct Eight {
  float x[8];
};

template <int TYPE>
__device__ __forceinline__ Eight load8(const void* p, float scale) {
  Eight r;
  if constexpr (TYPE == kBf16) {
    const uint4 u = *static_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.x[2 * i] = __uint_as_float(w[i] << 16);
      r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else if constexpr (TYPE == kF32) {
    const f32x4 lo = static_cast<const f32x4*>(p)[0], hi = static_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.x[i] = lo[i]; r.x[4 + i] = hi[i]; }
  } else {
    const uint2 u = *static_cast<const uint2*>(p);
    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
      r.x[4 * i] = lo[0] * scale; r.x[4 * i + 1] = lo[1] * scale;
      r.x[4 * i + 2] = hi[0] * scale; r.x[4 * i + 3] = hi[1] * scale;
    }
  }
  return r;
}

template <int TYPE>
__device__ __forceinline__ void store8(void* p, const Eight& r) {
  if constexpr (TYPE == kBf16) {
    *static_cast<bf16x8*>(p) = pack8(r.x[0], r.x[1], r.x[2], r.x[3], r.x[4], r.x[5], r.x[6], r.x[7]);
  } else if constexpr (TYPE == kF32) {
    static_cast<f32x4*>(p)[0] = f32x4{r.x[0], r.x[1], r.x[2], r.x[3]};
    static_cast<f32x4*>(p)[1] = f32x4{r.x[4], r.x[5], r.x[6], r.x[7]};
  } else {
    uint2 u;
    u.x = __builtin_amdgcn_cvt_pk_fp8_f32(r.x[0], r.x[1], 0, false);
    u.x = __builtin_amdgcn_cvt_pk_fp8_f32(r.x[2], r.x[3], u.x, true);
    u.y = __builtin_amdgcn_cvt_pk_fp8_f32(r.x[4], r.x[5], 0, false);
    u.y = __builtin_amdgcn_cvt_pk_fp8_f32(r.x[6], r.x[7], u.y, true);
    *static_cast<uint2*>(p) = u;
  }
}

constexpr int kBytes[3] = {2, 4, 1};

// Biased exponent of a row from the bits of its lanes' largest finite |x| (LANES lanes a row).  amax = m 2^x:
// e = x - 8, and one more where m is over 1.75 = 448 / 256.
template <int LANES>
__device__ __forceinline__ int row_exponent(const Eight& r) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {   // by the bits: this build's floating-point flags know no NaN
    const uint32_t u = __float_as_uint(r.x[i]) & 0x7fffffffu;
    top = max(top, u < 0x7f800000u ? u : 0u);
  }
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  return min(max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 17), 247);
}

// Infinities as NaN (a product with a power of two leaves them, and the conversion would saturate).
__device__ __forceinline__ float no_inf(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x7fffffffu) == 0x7f800000u ? __uint_as_float(u | 0x400000u) : x;
}

// The values of a row as the cache stores and reads them: the types' copy, or quantised.
constexpr int kSteps = 4;   // of 64 lanes, in flight together

template <int D, int ROWS, int CACHE, bool WRITE>
__global__ void __launch_bounds__(256) cache_kernel(PArgs a, int tokens, int waves_per_token, Div by_waves, int first_block) {
  constexpr int kLanes = D / 8;
  const int lane = thread_id() & 63, wave = uni((first_block + block_id()) * 4 + (thread_id() >> 6));
  const int unit = quot(wave, by_waves);                 // `tokens` tokens
  const int part = wave - unit * waves_per_token;
  const int t0 = unit * tokens;
  if (t0 >= a.T) return;
  const int items = 2 * a.Hkv * kLanes;                  // 8-value pieces of a token

  // this lane's pieces, and the call's rows
  int t[kSteps], c[kSteps], chunk[kSteps];
  bool is_v[kSteps], on[kSteps];
  Eight x[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    int i = (part * kSteps + s) * 64 + lane;
    t[s] = t0;
    if (tokens > 1) {                                    // items divides 64: 16 or 32
      t[s] += i / items;
      i &= items - 1;
    }
    on[s] = (tokens > 1 ? (part * kSteps + s) * 64 + lane < tokens * items : i < items) && t[s] < a.T;
    const int row = i / kLanes;
    chunk[s] = i % kLanes;
    is_v[s] = row >= a.Hkv;
    c[s] = is_v[s] ? row - a.Hkv : row;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[s].x[e] = 0.f;
    if (WRITE && on[s]) {
      const long long off = is_v[s] ? t[s] * a.v_t + c[s] * a.v_h : t[s] * a.k_t + c[s] * a.k_h;
      x[s] = load8<ROWS>(static_cast<const char*>(is_v[s] ? a.v : a.k) + (off + chunk[s] * 8) * kBytes[ROWS], 1.f);
    }
  }

  // the sequences of the tokens, one search for the wave where it has one token
  int b[kSteps];
  if (tokens == 1) {
    const int one = find_seq<-1>(a, t0, lane);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) b[s] = one;
  } else {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) b[s] = -1;
    for (int u = 0; u < tokens && t0 + u < a.T; ++u) {
      const int one = find_seq<-1>(a, t0 + u, lane);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) b[s] = t[s] == t0 + u ? one : b[s];
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    CacheRow at{-1, 0};
    bool mine = false;
    if (on[s] && b[s] >= 0) {
      const SeqRows sr = seq_rows(a, b[s]);
      mine = t[s] >= sr.s0 && t[s] < sr.s0 + sr.n;       // else: a row of no sequence
      if (mine) at = cache_row(a, b[s], sr.kv - sr.n + t[s] - sr.s0, sr.keys);
    }
    const long long cp = is_v[s] ? a.vc_p : a.kc_p, ct = is_v[s] ? a.vc_t : a.kc_t, ch = is_v[s] ? a.vc_h : a.kc_h;
    char* cached = (is_v[s] ? a.vc : a.kc) + (at.page * cp + at.at * ct + c[s] * ch + chunk[s] * 8) * kBytes[CACHE];
    uint8_t* exps = nullptr;
    if constexpr (CACHE == kE4m3)
      exps = is_v[s] ? a.ve + at.page * a.ve_p + at.at * a.ve_t + c[s] * a.ve_h : a.ke + at.page * a.ke_p + at.at * a.ke_t + c[s] * a.ke_h;
    if constexpr (WRITE) {
      if constexpr (CACHE == kE4m3) {
        const int e = row_exponent<kLanes>(x[s]);        // all lanes of a row are here together
        const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[s].x[i] = no_inf(x[s].x[i] * inv);
        if (at.page >= 0 && chunk[s] == 0) *exps = (uint8_t)e;
      }
      if (at.page >= 0) store8<CACHE>(cached, x[s]);
    } else if (mine) {
      Eight y;
#pragma unroll
      for (int i = 0; i < 8; ++i) y.x[i] = 0.f;          // no such position, or no page: zeros
      if (at.page >= 0) {
        float scale = 1.f;
        if constexpr (CACHE == kE4m3) scale = __uint_as_float((uint32_t)*exps << 23);
        y = load8<CACHE>(cached, scale);
      }
      const long long off = is_v[s] ? t[s] * a.v_t + c[s] * a.v_h : t[s] * a.k_t + c[s] * a.k_h;
      store8<ROWS>(static_cast<char*>(is_v[s] ? a.v : a.k) + (off + chunk[s] * 8) * kBytes[ROWS], y);
    }
  }
}

template <int D, int ROWS, int CACHE, bool WRITE>
int launch(const PArgs& a, hipStream_t st) {
  const int items = 2 * a.Hkv * (D / 8);
  const int tokens = items < 64 ? 64 / items : 1;
  const int waves = (items * tokens + 64 * kSteps - 1) / (64 * kSteps);
  const long long total = (long long)((a.T + tokens - 1) / tokens) * waves;
  return launch_blocks(cache_kernel<D, ROWS, CACHE, WRITE>, (int)((total + 3) / 4), 256, st, a, tokens, waves, div_by(waves));
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
