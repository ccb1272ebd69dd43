// fp32 attention of new tokens over a paged cache (fp32 or e4m3), and the joining of pieces for both row types.
//
// The rows and the walk are those of the bf16 kernel, in workgroups of 64 rows and tiles of 32 keys; the arithmetic is that of
// the fp32 kernels on contiguous tensors (v_mfma_f32_16x16x4_f32).  One token over 256 keys, four heads: 8.2 us, what a CU needs to
// fetch one head's K and V by itself (64 keys: 5.1 us); one token of 16 sequences over 8000, H = 8, D = 128: 180 us, 5.8 TB/s.
#include <cfloat>

#include "s2attn_f32_tile.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

constexpr int kRowsLog2 = 6;
static_assert(kWgRows == 1 << kRowsLog2, "rows of a workgroup");

template <int D, bool E4M3>
__device__ __forceinline__ void chunk_f32_workgroup(const PArgs& a, int block, char* smem) {   // smem: [stage][K, V]
  using L = Lanes<D>;
  constexpr int kEsz = E4M3 ? 1 : 4;

  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int c16 = lane & 15, q4 = lane >> 4;
  int tile, c, split;
  if (!tile_of_block(a, a.chunk, block, tile, c, split)) return;
  const SeqRows sr = find_rows<kRowsLog2>(a, tile, lane);
  const int b = sr.b;
  if (b < 0) return;
  const int i0 = uni((tile - first_tile<kRowsLog2>(a, sr.s0, b)) * kWgRows), n_rows = uni(sr.n * a.r);
  if (i0 < 0 || i0 >= n_rows || n_rows <= a.few_rows) return;   // (less than 0: row_start falls somewhere)
  const int p_first = uni(sr.kv - sr.n);
  const int p_lo = uni(p_first + quot(i0, a.by_r));
  const int p_hi = uni(p_first + quot(min(i0 + kWgRows, n_rows) - 1, a.by_r));
  const KeyTiles kt = key_tiles<kTile>(a.window, a.sinks, p_lo, p_hi, sr.keys);
  const Piece piece = pieces_of(a.chunk, kt.total);
  const int per = piece.per, n0 = split * per, n1 = uni(min(kt.total, n0 + per));
  if (split > 0 && n0 >= n1) return;

  const int iw = i0 + 16 * w, row = min(iw + c16, n_rows - 1);
  const int tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
  const int t = sr.s0 + tq, pos = min(p_first + tq, sr.keys - 1), n_seen = keys_up_to(a.window, p_first + tq, pos);
  const int w_lo = uni(p_first + quot(min(iw, n_rows - 1), a.by_r));
  const int w_hi = uni(p_first + quot(min(iw + 16, n_rows) - 1, a.by_r));
  const bool idle = iw >= n_rows;
  const float c2 = a.scale_log2;

  const uint64_t k_head = reinterpret_cast<uint64_t>(a.kc) + c * a.kc_h * kEsz;
  const uint64_t v_head = reinterpret_cast<uint64_t>(a.vc) + c * a.vc_h * kEsz;
  const uint64_t ke_head = reinterpret_cast<uint64_t>(a.ke) + c * a.ke_h, ve_head = reinterpret_cast<uint64_t>(a.ve) + c * a.ve_h;
  const uint32_t base = lds_addr(smem);
  // every wave looks up the 32 keys of a tile, twice; `seen` has a bit for each that exists and that some row sees
  auto look_up = [&](int n) __attribute__((always_inline)) {
    const int j = kt.tile(n) * kTile + (lane & 31);
    return cache_row(a, b, j, n < n1 && is_seen(a, p_lo, kt.end, j));
  };
  auto seen_of = [&](const CacheRow& x) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_ballot_w64(x.page >= 0); };

  L ln;
  ln.init(lane, w);
  constexpr int kLoads = kTile * (D / 16) / 256 > 0 ? kTile * (D / 16) / 256 : 1;   // e4m3: 16-value loads of a thread
  constexpr bool kAll = kTile * (D / 16) >= 256;                                    // else the upper half of the threads has none
  u32x4 k8[kLoads], v8[kLoads];
  float ks8[kLoads], vs8[kLoads];
  auto issue = [&](const CacheRow& x, int stage) __attribute__((always_inline)) {
    const uint32_t dst = base + stage * 2 * L::kTileBytes;
    if constexpr (!E4M3) {
      constexpr int kStep = 4 * (64 / (D / 4));    // rows the four waves fill together: 16 or 8
#pragma unroll
      for (int p = 0; p < kTile / kStep; ++p) {
        const int rr = p * kStep + ln.st_row;
        const int page = __shfl(x.page, rr), at = __shfl(x.at, rr);
        const uint64_t zero = zero_address();
        const uint64_t ks = page < 0 ? zero : k_head + (page * a.kc_p + at * a.kc_t) * 4;
        const uint64_t vs = page < 0 ? zero : v_head + (page * a.vc_p + at * a.vc_t) * 4;
        dma16(reinterpret_cast<const void*>(ks + (ln.st_chunk << 4)), dst + (p * 4 + w) * 1024);
        dma16(reinterpret_cast<const void*>(vs + (ln.st_chunk << 4)), dst + (p * 4 + w) * 1024 + L::kTileBytes);
      }
    } else {
#pragma unroll
      for (int p = 0; p < kLoads; ++p) {
        const int i = p * 256 + tid, rr = i / (D / 16), chunk = i % (D / 16);
        const int page = __shfl(x.page, rr & 31), at = __shfl(x.at, rr & 31);
        const uint64_t zero = zero_address();
        const bool there = page >= 0 && (kAll || rr < kTile);
        k8[p] = load16((there ? k_head + page * a.kc_p + at * a.kc_t : zero) + chunk * 16);
        v8[p] = load16((there ? v_head + page * a.vc_p + at * a.vc_t : zero) + chunk * 16);
        ks8[p] = load_scale(there ? ke_head + page * a.ke_p + at * a.ke_t : zero);
        vs8[p] = load_scale(there ? ve_head + page * a.ve_p + at * a.ve_t : zero);
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
            const u32x4 u = kv ? v8[p] : k8[p];
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
      const bool masked = j0 + kTile - 1 > w_lo || ~seen != 0 || (a.window > 0 && j0 < w_hi - a.window + 1);
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) sc[kb] *= c2;
      if (masked) {
        int d0 = pos - j0 - 4 * q4;
        asm volatile("" : "+v"(d0));   // keeps the compiler from doing this ahead of the branch
        const int last = min(pos, (a.window > 0 ? a.sinks : 0) - 1) - j0 - 4 * q4;
        const uint32_t seen_l = seen >> (4 * q4);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int bit = 16 * kb + v;
            const bool in = (((unsigned)(d0 - bit) < (unsigned)n_seen) | (bit <= last)) & (seen_l >> bit & 1);
            sc[kb][v] = in ? sc[kb][v] : -INFINITY;
          }
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sc[kb][v]);
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
  const PArgs z = late_args();
  const int H = z.Hkv * z.r;
  if (piece.count > 1) {
    const size_t at = part_row(z, z.chunk, false, split, b, c, 0, t, h);
    store_row<D>(z.chunk.part_o + at * D, o, inv, q4);
    if (q4 == 0) z.chunk.part_lse[at] = lse2;
    return;
  }
  store_row<D>(static_cast<float*>(z.o) + ((size_t)t * H + h) * D, o, inv, q4);
  if (q4 == 0 && z.lse) z.lse[(size_t)h * z.T + t] = lse2 * kLn2;
}

// ---- few rows: sixteen rows of a sequence at a time, the waves on different tiles of 16 keys, K and V straight to registers, the next
// tile on its way while one is worked on (as in the bf16 kernel; operands as in s2attn_f32_small.hip).
//   K  lane (c16, q4) has key c16: fp32 floats 16 i + 4 q4 .., e4m3 values 16 (q4 + 4 i) ..; Q agrees
//   V  lane (c16, q4) has keys 4 q4 + v, values 64 j + 4 c16 ..
template <int D, bool E4M3>
struct FewTile {
  u32x4 k[E4M3 ? D / 64 : D / 16];
  uint32_t v8[4][D / 64];
  f32x4 v[4][D / 64];
  float ks, vs[4];
  uint32_t seen;
};

template <int D, bool E4M3, bool BOTH>   // BOTH: beside the other kind of workgroup
__device__ __forceinline__ void few_f32_workgroup(const PArgs& a, int block, float* blocks, float (*max_s)[16], float (*sum_s)[16]) {
  using T = FewTile<D, E4M3>;
  constexpr int TK = 16, kWaves = 4, kEsz = E4M3 ? 1 : 4, kStride = D + 4;
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int c16 = lane & 15, q4 = lane >> 4;
  const int y = quot(block, a.by_Hkv), c = block - y * a.Hkv;
  const int unit = quot(y, a.few.by_splits), split = y - unit * a.few.splits;
  FewRows rows;
  if (!few_rows_of<BOTH>(a, unit, lane, rows)) return;
  const SeqRows sr = rows.sr;
  const int b = sr.b, n_rows = rows.i1, p_first = uni(sr.kv - sr.n);
  const uint64_t k_head = reinterpret_cast<uint64_t>(a.kc) + c * a.kc_h * kEsz + 16 * q4;
  const uint64_t v_head = reinterpret_cast<uint64_t>(a.vc) + c * a.vc_h * kEsz + 4 * c16 * kEsz;
  const uint64_t ke_head = reinterpret_cast<uint64_t>(a.ke) + c * a.ke_h, ve_head = reinterpret_cast<uint64_t>(a.ve) + c * a.ve_h;
  const float c2 = a.scale_log2;

  for (int i0 = rows.i0; i0 < n_rows; i0 += 16) {
    const int p_lo = uni(p_first + quot(i0, a.by_r)), p_hi = uni(p_first + quot(min(i0 + 16, n_rows) - 1, a.by_r));
    const KeyTiles kt = key_tiles<TK>(a.window, a.sinks, p_lo, p_hi, sr.keys);
    const Piece piece = pieces_of(a.few, kt.total);
    const int n0 = split * piece.per, n1 = uni(min(kt.total, n0 + piece.per));
    if (split > 0 && n0 >= n1) continue;

    auto look_up = [&](int n) __attribute__((always_inline)) {
      const int j = kt.tile(n) * TK + c16;
      return cache_row(a, b, j, n < n1 && is_seen(a, p_lo, kt.end, j));
    };
    auto load = [&](T& t, const CacheRow& x) __attribute__((always_inline)) {
      t.seen = (uint32_t)__builtin_amdgcn_ballot_w64(x.page >= 0) & 0xffffu;
      const uint64_t zero = zero_address();
      const uint64_t kp = x.page >= 0 ? k_head + (x.page * a.kc_p + x.at * a.kc_t) * kEsz : zero;
#pragma unroll
      for (int i = 0; i < (E4M3 ? D / 64 : D / 16); ++i) t.k[i] = load16(kp + 64 * i);
      if constexpr (E4M3) t.ks = load_scale(x.page >= 0 ? ke_head + x.page * a.ke_p + x.at * a.ke_t : zero);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int page = __shfl(x.page, 4 * q4 + v), at = __shfl(x.at, 4 * q4 + v);
        const uint64_t vp = page >= 0 ? v_head + (page * a.vc_p + at * a.vc_t) * kEsz : zero;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          if constexpr (E4M3) t.v8[v][j] = S2_GLOBAL(uint32_t, vp + 64 * j);
          else t.v[v][j] = S2_GLOBAL(f32x4, vp + 256 * j);
        }
        if constexpr (E4M3) t.vs[v] = load_scale(page >= 0 ? ve_head + page * a.ve_p + at * a.ve_t : zero);
      }
    };
    auto widen4 = [](uint32_t u, float s) __attribute__((always_inline)) {
      const auto l = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), g = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
      return f32x4{l[0] * s, l[1] * s, g[0] * s, g[1] * s};
    };

    // the look-up of a tile goes out ahead of the loads of the tile before it, so that waiting for it is not waiting for them
    T ta, tb;
    CacheRow at = look_up(n0 + w), at_next = look_up(n0 + w + kWaves);
    load(ta, at);
    const int row = min(i0 + c16, n_rows - 1), tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
    const int pos = min(p_first + tq, sr.keys - 1), n_seen = keys_up_to(a.window, p_first + tq, pos), t = sr.s0 + tq;
    f32x4 qf[D / 16];
    {
      const float* q = static_cast<const float*>(a.q) + t * a.q_t + h * a.q_h;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        qf[i] = *reinterpret_cast<const f32x4*>(q + (E4M3 ? 16 * (q4 + 4 * (i >> 2)) + 4 * (i & 3) : 16 * i + 4 * q4));
    }
    f32x4 o[D / 64][4];
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -FLT_MAX, l_run = 0.f;

    auto step = [&](T& cur, T& nxt, int n) __attribute__((always_inline)) {
      at = at_next;
      at_next = look_up(n + 2 * kWaves);
      load(nxt, at);
      const int j0 = kt.tile(n) * TK;
      f32x4 sc = {0.f, 0.f, 0.f, 0.f}, odd = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        f32x4 x;
        if constexpr (E4M3) {
          const u32x4 u = cur.k[i >> 2];
          x = widen4((i & 3) == 0 ? u.x : (i & 3) == 1 ? u.y : (i & 3) == 2 ? u.z : u.w, cur.ks);
        } else {
          x = __builtin_bit_cast(f32x4, cur.k[i]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (i & 1) odd = mfma4(x[e], qf[i][e], odd);
          else sc = mfma4(x[e], qf[i][e], sc);
        }
      }
      sc += odd;
      const bool masked = j0 + TK - 1 > p_lo || cur.seen != 0xffffu || (a.window > 0 && j0 < p_hi - a.window + 1);
      float mx = -INFINITY;
      sc *= c2;
      if (masked) {
        int d0 = pos - j0 - 4 * q4;
        asm volatile("" : "+v"(d0));
        const int last = min(pos, (a.window > 0 ? a.sinks : 0) - 1) - j0 - 4 * q4;
        const uint32_t seen_l = cur.seen >> (4 * q4);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const bool in = (((unsigned)(d0 - v) < (unsigned)n_seen) | (v <= last)) & (seen_l >> v & 1);
          sc[v] = in ? sc[v] : -INFINITY;
        }
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sc[v]);
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
      for (int v = 0; v < 4; ++v) {
        sc[v] = exp2f(sc[v] - m_run);
        l_run += sc[v];
      }
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          f32x4 x;
          if constexpr (E4M3) x = widen4(cur.v8[v][j], cur.vs[v]);
          else x = cur.v[v][j];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][e] = mfma4(x[e], sc[v], o[j][e]);
        }
    };
    for (int n = n0 + w; n < n1; n += 2 * kWaves) {
      step(ta, tb, n);
      if (n + kWaves < n1) step(tb, ta, n + kWaves);
    }

    const PArgs z = BOTH ? late_args() : a;
    l_run = sum_cols(l_run);
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<f32x4*>(blocks + (w * 16 + c16) * kStride + 64 * j + 16 * q4 + 4 * x) = f32x4{o[j][0][x], o[j][1][x], o[j][2][x], o[j][3][x]};
    if (q4 == 0) {
      max_s[w][c16] = m_run;
      sum_s[w][c16] = l_run;
    }
    __syncthreads();
    constexpr int kLanes = D / 8;   // 8 columns a thread: 16 or 32 rows at once
    const int r16 = tid / kLanes, ch = tid % kLanes;
    if (r16 < 16 && i0 + r16 < n_rows) {
      float m = max_s[0][r16], l = 0.f;
#pragma unroll
      for (int x = 1; x < kWaves; ++x) m = fmaxf(m, max_s[x][r16]);
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float f = exp2f(max_s[x][r16] - m);
        l = fmaf(sum_s[x][r16], f, l);
        const f32x4* p = reinterpret_cast<const f32x4*>(blocks + (x * 16 + r16) * kStride + 8 * ch);
        s0 += p[0] * f;
        s1 += p[1] * f;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
      const int ti = quot(i0 + r16, z.by_r), hi = c * z.r + i0 + r16 - ti * z.r, tt = sr.s0 + ti, H = z.Hkv * z.r;
      float* dst;
      if (piece.count > 1) {
        const size_t at2 = part_row(z, z.few, z.few_slots, split, b, c, i0 + r16, tt, hi);
        dst = z.few.part_o + at2 * D;
        if (ch == 0) z.few.part_lse[at2] = lse2;
      } else {
        dst = static_cast<float*>(z.o) + ((size_t)tt * H + hi) * D;
        if (ch == 0 && z.lse) z.lse[(size_t)hi * z.T + tt] = lse2 * kLn2;
      }
      *reinterpret_cast<f32x4*>(dst + 8 * ch) = s0 * inv;
      *reinterpret_cast<f32x4*>(dst + 8 * ch + 4) = s1 * inv;
    }
    __syncthreads();   // before the next rows' sums
  }
}

template <int D>
constexpr int kChunkBytes = 4 * Lanes<D>::kTileBytes;
template <int D>
constexpr int kFewBytes = 4 * 16 * (D + 4) * 4;

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_f32_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kChunkBytes<D>];
  chunk_f32_workgroup<D, E4M3>(a, first_block + block_id(), smem);
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_few_f32_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(16))) float blocks[kFewBytes<D> / 4];
  __shared__ float max_s[4][16], sum_s[4][16];
  few_f32_workgroup<D, E4M3, false>(a, first_block + block_id(), blocks, max_s, sum_s);
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_both_f32_kernel(PArgs a, int first_block) {
  static_assert(kFewBytes<D> <= kChunkBytes<D>, "one room for both");
  __shared__ __attribute__((aligned(1024))) char smem[kChunkBytes<D>];
  __shared__ float max_s[4][16], sum_s[4][16];
  const int block = first_block + block_id();
  if (block < a.chunk_blocks)
    chunk_f32_workgroup<D, E4M3>(a, block, smem);
  else
    few_f32_workgroup<D, E4M3, true>(a, block - a.chunk_blocks, reinterpret_cast<float*>(smem), max_s, sum_s);
}

// o = sum of the pieces' outputs by their share exp2(lse_s - lse) of the row.  D / 4 lanes hold a piece's output; G groups of so
// many lanes take the pieces of one row, four at a time (each group with a running maximum of its own), the other groups of a
// workgroup other heads of the same token, `heads` of them to a workgroup.  Bound by latency: six workgroups to a CU hide it
// better than the four that the compiler would have left room for (13.4 and 11.2 us for the case below).
// FEW: only sequences of `few` are in pieces, in slots, and of each only the first per_seq tokens are looked at.
template <int D, int TK, int FEW_TK, bool BF16, bool FEW>
__global__ void __launch_bounds__(256, 6) paged_join_kernel(PArgs a, int nq, int heads, int head_blocks, Div by_head_blocks, int per_seq,
                                                            Div by_seq, int first_block) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ float4 acc_s[kGroups][kLanes];
  __shared__ float m_s[kGroups], l_s[kGroups];
  const int tid = thread_id(), H = a.Hkv * a.r;
  const int block = first_block + block_id(), unit = quot(block, by_head_blocks), h0 = (block - unit * head_blocks) * heads;
  int t = unit;
  SeqRows sr;
  if constexpr (FEW) {
    const int b = quot(unit, by_seq);
    if (b >= a.B) return;
    sr = seq_rows(a, b);
    t = sr.s0 + unit - b * per_seq;
  } else {
    if (t >= a.T) return;
    sr = find_rows<-1>(a, t, tid & 63);
  }
  if (sr.b < 0 || t < sr.s0 || t >= sr.s0 + sr.n) return;
  const int tok = t - sr.s0, p_first = sr.kv - sr.n, first = quot(tok, a.by_few_tokens) * a.few_tokens;
  const bool few = sr.n * a.r <= a.few_rows;
  if (FEW && !few) return;
  const int i0 = first * a.r, i1 = min(first + a.few_tokens, sr.n) * a.r;   // the rows that were dealt out with it
  const int tile = few ? 16 * nq : a.chunk_rows;
  const PSet& set = few ? a.few : a.chunk;
  if (set.splits == 1) return;                    // in one piece: written by the attention kernel
  const int log2g = set.splits <= 4 ? 0 : set.splits <= 8 ? 1 : set.splits <= 16 ? 2 : 3;
  const int g = tid / kLanes, l = tid % kLanes, sub = g >> log2g, piece0 = g & ((1 << log2g) - 1);
  const size_t step = set.part_rows;
  for (int hh = 0; hh < heads; hh += kGroups >> log2g) {
    const int h = h0 + hh + sub;
    const bool on = hh + sub < heads && h < H;
    const int i = tok * a.r + (h - quot(h, a.by_r) * a.r), j0 = i0 + ((i - i0) & ~(tile - 1));   // tile: a power of two
    const int p_lo = p_first + quot(j0, a.by_r), p_hi = p_first + quot(min(j0 + tile, i1) - 1, a.by_r);
    const KeyTiles kt = few ? key_tiles<FEW_TK>(a.window, a.sinks, p_lo, p_hi, sr.keys) : key_tiles<TK>(a.window, a.sinks, p_lo, p_hi, sr.keys);
    const Piece piece = pieces_of(set, kt.total);
    const int pieces = on && piece.count > 1 ? piece.count : 0;
    const size_t row = part_row(a, set, FEW || (few && a.few_slots), 0, sr.b, quot(h, a.by_r), i, t, h);
    const float* po = set.part_o + row * D + 4 * l;
    const float* pl = set.part_lse + row;
    float m = -FLT_MAX, sum = 0.f;
    float4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = piece0; s0 < pieces; s0 += 4 << log2g) {
      float ls[4];
      float4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = s0 + (u << log2g);
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
    if (log2g > 0) {
      acc_s[g][l] = acc;
      if (l == 0) { m_s[g] = m; l_s[g] = sum; }
      __syncthreads();
      if (piece0 == 0) {
        float top = m;
        for (int x = 1; x < 1 << log2g; ++x) top = fmaxf(top, m_s[g + x]);
        sum = 0.f;
        acc = float4{0.f, 0.f, 0.f, 0.f};
        for (int x = 0; x < 1 << log2g; ++x) {
          const float f = exp2f(m_s[g + x] - top);
          sum = fmaf(l_s[g + x], f, sum);
          acc.x = fmaf(acc_s[g + x][l].x, f, acc.x); acc.y = fmaf(acc_s[g + x][l].y, f, acc.y);
          acc.z = fmaf(acc_s[g + x][l].z, f, acc.z); acc.w = fmaf(acc_s[g + x][l].w, f, acc.w);
        }
        m = top;
      }
      __syncthreads();   // before the next heads' sums
    }
    if (piece0 != 0 || pieces == 0) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t at = ((size_t)t * H + h) * D + 4 * l;
    if constexpr (BF16)
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.o) + at) = pack4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    else
      *reinterpret_cast<float4*>(static_cast<float*>(a.o) + at) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (l == 0 && a.lse) a.lse[(size_t)h * a.T + t] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
  }
}

template <int D, int TK, int FEW_TK, bool BF16>
int join_t(const PArgs& a, int nq, hipStream_t st) {
  constexpr int kGroups = 1024 / D;
  const int H = a.Hkv * a.r, splits = a.few.splits > a.chunk.splits ? a.few.splits : a.chunk.splits;
  const int per_seq = a.few_slots && a.chunk.splits == 1 ? a.few_rows / a.r : 0, units = per_seq > 0 ? a.B * per_seq : a.T;
  // heads go together while 2048 workgroups are left: 16 sequences of 1 to 600 rows, H = 32, D = 64, down to 512, 2048 and 4096
  // 20, 10.0 and 11.2 us
  int heads = splits <= 4 ? kGroups : splits <= 8 ? kGroups / 2 : splits <= 16 ? kGroups / 4 : kGroups / 8;
  while (2 * heads <= H && (long long)units * (H / (2 * heads)) >= 2048) heads *= 2;
  const int head_blocks = (H + heads - 1) / heads;
  auto launch = [&](auto kernel) {
    return launch_blocks(kernel, units * head_blocks, 256, st, a, nq, heads, head_blocks, div_by(head_blocks), per_seq, div_by(per_seq > 0 ? per_seq : 1));
  };
  return per_seq > 0 ? launch(paged_join_kernel<D, TK, FEW_TK, BF16, true>) : launch(paged_join_kernel<D, TK, FEW_TK, BF16, false>);
}

template <int D, bool E4M3>
int launch_pages(const PArgs& a, hipStream_t st) {
  const int few = a.few.n_tiles * a.Hkv * a.few.splits;
  if (a.chunk_blocks == 0) return launch_blocks(paged_few_f32_kernel<D, E4M3>, few, 256, st, a);
  if (a.few_rows == 0) return launch_blocks(paged_f32_kernel<D, E4M3>, a.chunk_blocks, 256, st, a);
  return launch_blocks(paged_both_f32_kernel<D, E4M3>, a.chunk_blocks + few, 256, st, a);
}

}  // namespace

int launch_paged_f32(const PArgs& a, int D, bool e4m3, hipStream_t st) {
  if (D == 64) return e4m3 ? launch_pages<64, true>(a, st) : launch_pages<64, false>(a, st);
  return e4m3 ? launch_pages<128, true>(a, st) : launch_pages<128, false>(a, st);
}

int launch_paged_join(const PArgs& a, int D, bool bf16, int nq, hipStream_t st) {
  if (bf16) return D == 64 ? join_t<64, 64, 32, true>(a, nq, st) : join_t<128, 64, 32, true>(a, nq, st);
  return D == 64 ? join_t<64, 32, 16, false>(a, nq, st) : join_t<128, 32, 16, false>(a, nq, st);
}

}  // namespace s2
