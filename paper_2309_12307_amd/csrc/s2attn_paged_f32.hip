// fp32 attention of new tokens over a paged cache (fp32 or e4m3), and the joining of pieces for both row types.
//
// The rows and the walk are those of the bf16 kernel, in workgroups of 64 rows and tiles of 32 keys; the arithmetic is that of
// the fp32 kernels on contiguous tensors (v_mfma_f32_16x16x4_f32).
#include <cfloat>

#include "s2attn_f32_tile.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

constexpr int kRowsLog2 = 6;
static_assert(kWgRows == 1 << kRowsLog2, "rows of a workgroup");

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_f32_kernel(PArgs a, int first_block) {
  using L = Lanes<D>;
  constexpr int kEsz = E4M3 ? 1 : 4;
  __shared__ __attribute__((aligned(1024))) char smem[4 * L::kTileBytes];   // [stage][K, V]

  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int c16 = lane & 15, q4 = lane >> 4;
  int tile, c, split;
  if (!tile_of_block(a, first_block + block_id(), tile, c, split)) return;
  const int b = find_seq<kRowsLog2>(a, tile, lane);
  if (b < 0) return;
  const SeqRows sr = seq_rows(a, b);
  const int i0 = uni((tile - first_tile<kRowsLog2>(a, b)) * kWgRows), n_rows = uni(sr.n * a.r);
  if (i0 >= n_rows) return;
  const int p_first = uni(sr.kv - sr.n);
  const int p_lo = uni(p_first + quot(i0, a.by_r));
  const int p_hi = uni(p_first + quot(min(i0 + kWgRows, n_rows) - 1, a.by_r));
  const KeyTiles kt = key_tiles<kTile>(a.window, a.sinks, p_lo, p_hi, sr.keys);
  const int per = tiles_of_split(a, kt.total);
  const int n0 = split * per, n1 = uni(min(kt.total, n0 + per));
  if (split > 0 && n0 >= n1) return;

  const int iw = i0 + 16 * w, row = min(iw + c16, n_rows - 1);
  const int tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
  const int t = sr.s0 + tq, pos = min(p_first + tq, sr.keys - 1);
  const int w_lo = uni(p_first + quot(min(iw, n_rows - 1), a.by_r));
  const int w_hi = uni(p_first + quot(min(iw + 16, n_rows) - 1, a.by_r));
  const bool idle = iw >= n_rows;
  const float c2 = a.scale_log2;

  const char* k_head = a.kc + c * a.kc_h * kEsz;
  const char* v_head = a.vc + c * a.vc_h * kEsz;
  const uint32_t base = lds_addr(smem);
  // every wave looks up the 32 keys of a tile, twice; `seen` has a bit for each that exists
  auto look_up = [&](int n) __attribute__((always_inline)) {
    return n < n1 ? cache_row(a, b, kt.tile(n) * kTile + (lane & 31), kt.end) : CacheRow{-1, 0};
  };
  auto seen_of = [&](const CacheRow& x) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_ballot_w64(x.page >= 0); };

  L ln;
  ln.init(lane, w);
  constexpr int kLoads = kTile * (D / 16) / 256 > 0 ? kTile * (D / 16) / 256 : 1;   // e4m3: 16-value loads of a thread
  constexpr bool kAll = kTile * (D / 16) >= 256;                                    // else the upper half of the threads has none
  uint4 k8[kLoads], v8[kLoads];
  float ks8[kLoads], vs8[kLoads];
  auto issue = [&](const CacheRow& x, int stage) __attribute__((always_inline)) {
    const uint32_t dst = base + stage * 2 * L::kTileBytes;
    if constexpr (!E4M3) {
      constexpr int kStep = 4 * (64 / (D / 4));    // rows the four waves fill together: 16 or 8
#pragma unroll
      for (int p = 0; p < kTile / kStep; ++p) {
        const int rr = p * kStep + ln.st_row;
        const int page = __shfl(x.page, rr), at = __shfl(x.at, rr);
        const char* zero = reinterpret_cast<const char*>(zero_row);
        const char* ks = page < 0 ? zero : k_head + (page * a.kc_p + at * a.kc_t) * 4;
        const char* vs = page < 0 ? zero : v_head + (page * a.vc_p + at * a.vc_t) * 4;
        dma16(ks + (ln.st_chunk << 4), dst + (p * 4 + w) * 1024);
        dma16(vs + (ln.st_chunk << 4), dst + (p * 4 + w) * 1024 + L::kTileBytes);
      }
    } else {
#pragma unroll
      for (int p = 0; p < kLoads; ++p) {
        const int i = p * 256 + tid, rr = i / (D / 16), chunk = i % (D / 16);
        const int page = __shfl(x.page, rr & 31), at = __shfl(x.at, rr & 31);
        k8[p] = v8[p] = uint4{0, 0, 0, 0};
        ks8[p] = vs8[p] = 1.f;
        if (page >= 0 && (kAll || rr < kTile)) {
          k8[p] = *reinterpret_cast<const uint4*>(k_head + page * a.kc_p + at * a.kc_t + chunk * 16);
          v8[p] = *reinterpret_cast<const uint4*>(v_head + page * a.vc_p + at * a.vc_t + chunk * 16);
          ks8[p] = __uint_as_float((uint32_t)a.ke[page * a.ke_p + at * a.ke_t + c * a.ke_h] << 23);
          vs8[p] = __uint_as_float((uint32_t)a.ve[page * a.ve_p + at * a.ve_t + c * a.ve_h] << 23);
        }
      }
    }
  };
  auto land = [&](int stage) __attribute__((always_inline)) {
    if constexpr (E4M3) {
      char* dst = smem + stage * 2 * L::kTileBytes;
#pragma unroll
      for (int p = 0; p < kLoads; ++p) {
        const int i = p * 256 + tid, rr = i / (D / 16), chunk = i % (D / 16);
        if (kAll || rr < kTile) {
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint4 u = kv ? v8[p] : k8[p];
            const float s = kv ? vs8[p] : ks8[p];
            const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const auto l = __builtin_amdgcn_cvt_pk_f32_fp8(x[e], false), g = __builtin_amdgcn_cvt_pk_f32_fp8(x[e], true);
              *reinterpret_cast<f32x4*>(dst + kv * L::kTileBytes + rr * L::kRow + (((4 * chunk + e) ^ (rr & 7)) << 4)) =
                  f32x4{l[0] * s, l[1] * s, g[0] * s, g[1] * s};
            }
          }
        }
      }
    }
  };

  CacheRow next = look_up(n0);
  uint32_t seen = 0, seen_next = 0;
  if (n0 < n1) {
    seen_next = seen_of(next);
    issue(next, 0);
    land(0);
    next = look_up(n0 + 1);
  }
  f32x4 qf[D / 16];
  load_own<D>(qf, a.q, (size_t)(t * a.q_t + h * a.q_h), q4);
  f32x4 o[D / 64][4];
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -FLT_MAX, l_run = 0.f;   // base 2; finite: a row whose keys so far are all masked has weights of zero

  for (int n = n0; n < n1; ++n) {
    const int stage = (n - n0) & 1;
    wait_vmcnt0();
    __syncthreads();
    seen = seen_next;
    if (n + 1 < n1) {
      seen_next = seen_of(next);
      issue(next, stage ^ 1);
      next = look_up(n + 2);
    }
    const int j0 = kt.tile(n) * kTile;
    const bool skip = idle || j0 > w_hi || (a.window > 0 && j0 + kTile <= w_lo - a.window + 1 && j0 >= a.sinks);
    if (!skip) {
      const char* Ks = smem + stage * 2 * L::kTileBytes;
      const char* Vs = Ks + L::kTileBytes;
      f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
      scores<D>(sc, Ks, ln, qf);
      const bool windowed = a.window > 0 && j0 < w_hi - a.window + 1;
      const bool masked = j0 + kTile - 1 > w_lo || ~seen != 0 || windowed;
      const int first = windowed ? p_first + tq - a.window + 1 : 0;
      const uint32_t seen_l = seen >> (4 * q4);
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          float x = sc[kb][v] * c2;
          const int key = j0 + 16 * kb + 4 * q4 + v;
          if (masked && !(key <= pos && (key >= first || key < a.sinks) && (seen_l >> (16 * kb + v) & 1))) x = -INFINITY;
          sc[kb][v] = x;
          mx = fmaxf(mx, x);
        }
      mx = max_cols(mx);
      if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][e] *= alpha;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          sc[kb][v] = exp2f(sc[kb][v] - m_run);
          l_run += sc[kb][v];
        }
      accumulate<D>(o, Vs, ln, sc);
    }
    if (n + 1 < n1) land(stage ^ 1);
  }

  const float l_tot = sum_cols(l_run);
  if (iw + c16 >= n_rows) return;
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  const float lse2 = l_tot == 0.f ? -INFINITY : m_run + log2f(l_tot);
  const int H = a.Hkv * a.r;
  if (kt.total > per) {
    const size_t at = ((size_t)split * a.T + t) * H + h;
    store_row<D>(a.part_o + at * D, o, inv, q4);
    if (q4 == 0) a.part_lse[at] = lse2;
    return;
  }
  store_row<D>(static_cast<float*>(a.o) + ((size_t)t * H + h) * D, o, inv, q4);
  if (q4 == 0 && a.lse) a.lse[(size_t)h * a.T + t] = lse2 * kLn2;
}

// o = sum of the pieces' outputs by their share exp2(lse_s - lse) of the row, one workgroup to a row: D / 4 lanes hold a
// piece's output, so 8 or 16 pieces are in flight at a time, each group with a running maximum of its own.
template <int D, int SHIFT, int TK, bool BF16>
__global__ void __launch_bounds__(256) paged_join_kernel(PArgs a, Div by_H, int first_block) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ float4 acc_s[kGroups][kLanes];
  __shared__ float m_s[kGroups], l_s[kGroups];
  const int tid = thread_id(), H = a.Hkv * a.r;
  const int th = first_block + block_id(), t = quot(th, by_H), h = th - t * H;
  if (t >= a.T) return;
  const int b = find_seq<-1>(a, t, tid & 63);
  if (b < 0) return;
  const SeqRows sr = seq_rows(a, b);
  if (t >= sr.s0 + sr.n) return;
  const int i = (t - sr.s0) * a.r + (h - quot(h, a.by_r) * a.r), i0 = i & ~((1 << SHIFT) - 1);
  const int p_first = sr.kv - sr.n;
  const KeyTiles kt = key_tiles<TK>(a.window, a.sinks, p_first + quot(i0, a.by_r),
                                    p_first + quot(min(i0 + (1 << SHIFT), sr.n * a.r) - 1, a.by_r), sr.keys);
  const int per = tiles_of_split(a, kt.total);
  if (kt.total <= per) return;                    // in one piece: written by the attention kernel
  const int pieces = (kt.total + per - 1) / per;

  const int g = tid / kLanes, l = tid % kLanes;
  const size_t step = (size_t)a.T * H;
  const float* po = a.part_o + ((size_t)t * H + h) * D + 4 * l;
  const float* pl = a.part_lse + (size_t)t * H + h;
  float m = -FLT_MAX, sum = 0.f;
  float4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = g; s0 < pieces; s0 += 4 * kGroups) {
    float ls[4];
    float4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + u * kGroups;
      ls[u] = s < pieces ? pl[s * step] : -INFINITY;
      x[u] = s < pieces ? *reinterpret_cast<const float4*>(po + s * step * D) : float4{0.f, 0.f, 0.f, 0.f};
    }
    const float m_new = fmaxf(fmaxf(fmaxf(m, ls[0]), ls[1]), fmaxf(ls[2], ls[3]));
    const float alpha = exp2f(m - m_new);
    m = m_new;
    sum *= alpha;
    acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = exp2f(ls[u] - m);
      sum += f;
      acc.x = fmaf(x[u].x, f, acc.x); acc.y = fmaf(x[u].y, f, acc.y);
      acc.z = fmaf(x[u].z, f, acc.z); acc.w = fmaf(x[u].w, f, acc.w);
    }
  }
  acc_s[g][l] = acc;
  if (l == 0) { m_s[g] = m; l_s[g] = sum; }
  __syncthreads();
  if (g != 0) return;
  float top = m_s[0];
#pragma unroll
  for (int x = 1; x < kGroups; ++x) top = fmaxf(top, m_s[x]);
  float total = 0.f;
  acc = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < kGroups; ++x) {
    const float f = exp2f(m_s[x] - top);
    total = fmaf(l_s[x], f, total);
    acc.x = fmaf(acc_s[x][l].x, f, acc.x); acc.y = fmaf(acc_s[x][l].y, f, acc.y);
    acc.z = fmaf(acc_s[x][l].z, f, acc.z); acc.w = fmaf(acc_s[x][l].w, f, acc.w);
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  const size_t at = ((size_t)t * H + h) * D + 4 * l;
  if constexpr (BF16)
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.o) + at) = pack4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  else
    *reinterpret_cast<float4*>(static_cast<float*>(a.o) + at) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  if (l == 0 && a.lse) a.lse[(size_t)h * a.T + t] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
}

template <int D>
int launch_t(const PArgs& a, int cache, int blocks, hipStream_t st) {
  if (cache == 2) return launch_blocks(paged_f32_kernel<D, true>, blocks, 256, st, a);
  return launch_blocks(paged_f32_kernel<D, false>, blocks, 256, st, a);
}

}  // namespace

int launch_paged_f32(const PArgs& a, int D, int cache, int blocks, hipStream_t st) {
  return D == 64 ? launch_t<64>(a, cache, blocks, st) : launch_t<128>(a, cache, blocks, st);
}

int launch_paged_join(const PArgs& a, int D, bool bf16, hipStream_t st) {
  const int H = a.Hkv * a.r, rows = a.T * H;
  const Div by_H = div_by(H);
  if (bf16) {
    if (D == 64) return launch_blocks(paged_join_kernel<64, 7, 64, true>, rows, 256, st, a, by_H);
    return launch_blocks(paged_join_kernel<128, 7, 64, true>, rows, 256, st, a, by_H);
  }
  if (D == 64) return launch_blocks(paged_join_kernel<64, 6, 32, false>, rows, 256, st, a, by_H);
  return launch_blocks(paged_join_kernel<128, 6, 32, false>, rows, 256, st, a, by_H);
}

}  // namespace s2
