// bf16 attention of new tokens over a paged cache (bf16 or e4m3) for gfx950.
//
// The rows of one sequence and kv head are its (token, query head of the kv head) pairs, token by token, so that K and V
// are read once for all query heads that share them.  Two kinds of workgroup (4 waves) share a launch:
//   chunk  128 rows of a sequence that has many, and a piece of their keys; a wave owns 32 rows, the waves share the
//          64-key tiles, staged in LDS.  S^T = K Q^T, online softmax, O^T += V^T P^T as in the forward kernels on contiguous
//          tensors.  Bound by the matrix unit.
//   few    all rows of a sequence that has 16 or 32, as single tokens have, and a piece of its keys; the waves take different
//          32-key tiles and meet once, at the end.  Bound by HBM: what counts is bytes on the way, so a wave has a whole tile of
//          K and V on its way to registers while it works on another, and waits for nobody.
// Rows that several pieces share leave normalised fp32 partial outputs and their log-sum-exp, which a second kernel joins.
//
// P is rounded to bf16 for the second product (as everywhere in this library); the row sum adds the unrounded P, and
// statistics, outputs and partial outputs stay fp32 up to the one rounding of o.
#include "s2attn_bf16_fwd.h"
#include "s2attn_bf16_tile.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

constexpr int kKeys = 64;       // of a tile
constexpr int kRowsLog2 = 7;
constexpr int kRows = 1 << kRowsLog2;

// Removes the scores of keys that this lane's row does not see: after `pos`, before `first` and no sinks, or not there (`seen`: a
// bit a key, from this lane's first on, which is `key0`).
__device__ __forceinline__ void mask_paged(f32x16& s0, f32x16& s1, int key0, int pos, int first, int sinks, uint64_t seen) {
  const uint32_t seen0 = (uint32_t)seen, seen1 = (uint32_t)(seen >> 32);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int bit = 8 * (v >> 2) + (v & 3), key = key0 + bit;
    if (!(key <= pos && (key >= first || key < sinks) && (seen0 >> bit & 1))) s0[v] = -INFINITY;
    if (!(key + 32 <= pos && (key + 32 >= first || key + 32 < sinks) && (seen1 >> bit & 1))) s1[v] = -INFINITY;
  }
}

// A wave's 32 rows from iw on (lane l and l + 32: row l, token t and head h): o / l and the log-sum-exp, as a piece or as the
// output, the latter turned through the wave's part of LDS.  A row that saw nothing: 0 and -infinity.  m2: maximum, base 2.
template <int D>
__device__ __forceinline__ void chunk_epilogue(const PArgs& a, const f32x16 (&o)[D / 32], float m2, float l_run, char* region, int s0, int c,
                                               int iw, int n_rows, int t, int h, int split, int pieces, int lane) {
  using L = Tile<D>;
  constexpr int DB = D / 32, kChunks = D / 8, kRowsPer = 64 / kChunks;
  const int g32 = lane >> 5, l32 = lane & 31;
  const float l_tot = sum_halves(l_run);
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  const float lse2 = l_tot == 0.f ? -INFINITY : m2 + __builtin_amdgcn_logf(l_tot);
  const bool valid = iw + l32 < n_rows;
  const int H = a.Hkv * a.r;
  if (pieces > 1) {
    if (!valid) return;
    const size_t at = ((size_t)split * a.T + t) * H + h;
    float* dst = a.part_o + at * D + 4 * g32;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int vv = 0; vv < 4; ++vv)
        *reinterpret_cast<float4*>(dst + 32 * db + 8 * vv) =
            make_float4(o[db][4 * vv] * inv, o[db][4 * vv + 1] * inv, o[db][4 * vv + 2] * inv, o[db][4 * vv + 3] * inv);
    if (g32 == 0) a.part_lse[at] = lse2;
    return;
  }
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int vv = 0; vv < 4; ++vv)
      *reinterpret_cast<bf16x4*>(region + L::off(l32, 4 * db + vv) + 8 * g32) =
          pack4(o[db][4 * vv] * inv, o[db][4 * vv + 1] * inv, o[db][4 * vv + 2] * inv, o[db][4 * vv + 3] * inv);
  wave_lds_order();
  const int ch = lane % kChunks, sub = lane / kChunks;
  uint4 val[32 / kRowsPer];
#pragma unroll
  for (int it = 0; it < 32 / kRowsPer; ++it) val[it] = *reinterpret_cast<const uint4*>(region + L::off(it * kRowsPer + sub, ch));
#pragma unroll
  for (int it = 0; it < 32 / kRowsPer; ++it) {
    const int i = iw + it * kRowsPer + sub;
    if (i < n_rows) {
      const int ti = quot(i, a.by_r), hi = c * a.r + i - ti * a.r;
      *reinterpret_cast<uint4*>(static_cast<__bf16*>(a.o) + ((size_t)(s0 + ti) * H + hi) * D + ch * 8) = val[it];
    }
  }
  if (g32 == 0 && valid && a.lse) a.lse[(size_t)h * a.T + t] = lse2 * kLn2;
}

// smem: [stage][K, V]
template <int D, bool E4M3>
__device__ __forceinline__ void chunk_workgroup(const PArgs& a, int block, char* smem) {
  using L = Tile<D>;
  constexpr int kTileBytes = kKeys * L::kRow;
  constexpr int KS = D / 16, DB = D / 32, kChunks = D / 8;      // k-steps, column blocks, 16-byte chunks of a bf16 row
  constexpr int kEsz = E4M3 ? 1 : 2;
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  int tile, c, split;
  if (!tile_of_block(a, a.chunk, block, tile, c, split)) return;
  const int b = find_seq<kRowsLog2>(a, tile, lane);
  if (b < 0) return;
  const SeqRows sr = seq_rows(a, b);
  const int i0 = uni((tile - first_tile<kRowsLog2>(a, b)) * kRows), n_rows = uni(sr.n * a.r);
  if (i0 >= n_rows || n_rows <= a.few_rows) return;
  const int p_first = uni(sr.kv - sr.n);                        // position of the sequence's first row
  const int p_lo = uni(p_first + quot(i0, a.by_r));
  const int p_hi = uni(p_first + quot(min(i0 + kRows, n_rows) - 1, a.by_r));
  const KeyTiles kt = key_tiles<kKeys>(a.window, a.sinks, p_lo, p_hi, sr.keys);
  const Piece piece = pieces_of(a.chunk, kt.total);
  const int per = piece.per, n0 = split * per, n1 = uni(min(kt.total, n0 + per));
  if (split > 0 && n0 >= n1) return;                            // (the first piece also serves rows that see nothing)

  // this lane's row
  const int iw = i0 + 32 * w, row = min(iw + l32, n_rows - 1);
  const int tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
  const int t = sr.s0 + tq, pos = min(p_first + tq, sr.keys - 1);
  const int w_lo = uni(p_first + quot(min(iw, n_rows - 1), a.by_r));               // positions of the wave's rows
  const int w_hi = uni(p_first + quot(min(iw + 32, n_rows) - 1, a.by_r));
  const bool idle = iw >= n_rows;
  const float c2 = a.scale_log2;

  bf16x8 qf[KS];
  {
    const bf16x8* src = reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + t * a.q_t + h * a.q_h);
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = src[2 * k + g32];
  }

  const char* k_head = a.kc + c * a.kc_h * kEsz;
  const char* v_head = a.vc + c * a.vc_h * kEsz;
  const uint32_t smem_base = lds_addr(smem);
  // Every wave looks up all 64 keys of a tile, one a lane; `seen` has a bit for each that exists.
  auto look_up = [&](int n) __attribute__((always_inline)) {
    return n < n1 ? cache_row(a, b, kt.tile(n) * kKeys + lane, kt.end) : CacheRow{-1, 0};
  };
  auto seen_of = [&](const CacheRow& x) __attribute__((always_inline)) { return __builtin_amdgcn_ballot_w64(x.page >= 0); };

  // ---- staging.  bf16: global -> LDS, a lane's 16 bytes where the layout has the chunk; rows that are not there are
  // zeros.  e4m3: through registers, 16 values to two chunks.
  constexpr int kRowsPer = 64 / kChunks;                        // rows one wave instruction fills (bf16): 4 or 8
  constexpr int kPass = kKeys / (4 * kRowsPer);
  constexpr int kLoads = kKeys * (D / 16) / 256;                // 16-value loads of a thread and tensor (e4m3): 2 or 1
  uint4 k8[kLoads], v8[kLoads];
  float ks8[kLoads], vs8[kLoads];
  auto issue = [&](const CacheRow& x, int stage) __attribute__((always_inline)) {
    const uint32_t dst = smem_base + stage * 2 * kTileBytes;
    if constexpr (!E4M3) {
#pragma unroll
      for (int p = 0; p < kPass; ++p) {
        const int slot = (p * 4 + w) * 64 + lane;               // 16-byte slot of the tile in LDS
        int rr, chunk;
        if constexpr (D == 128) {
          rr = slot >> 4;
          chunk = (slot & 15) ^ swz(rr);
        } else {
          const int R = slot >> 4;
          rr = 2 * R + ((slot >> 3) & 1);
          chunk = (slot & 7) ^ swz64(R);
        }
        const int page = __shfl(x.page, rr), at = __shfl(x.at, rr);
        const char* zero = reinterpret_cast<const char*>(zero_row);
        const char* ks = page < 0 ? zero : k_head + (page * a.kc_p + at * a.kc_t) * 2;
        const char* vs = page < 0 ? zero : v_head + (page * a.vc_p + at * a.vc_t) * 2;
        dma16(ks + chunk * 16, dst + (p * 4 + w) * 1024);
        dma16(vs + chunk * 16, dst + (p * 4 + w) * 1024 + kTileBytes);
      }
    } else {
#pragma unroll
      for (int p = 0; p < kLoads; ++p) {
        const int i = p * 256 + tid, rr = i / (D / 16), chunk = i % (D / 16);
        const int page = __shfl(x.page, rr), at = __shfl(x.at, rr);
        k8[p] = v8[p] = uint4{0, 0, 0, 0};
        ks8[p] = vs8[p] = 1.f;
        if (page >= 0) {
          k8[p] = *reinterpret_cast<const uint4*>(k_head + page * a.kc_p + at * a.kc_t + chunk * 16);
          v8[p] = *reinterpret_cast<const uint4*>(v_head + page * a.vc_p + at * a.vc_t + chunk * 16);
          ks8[p] = __uint_as_float((uint32_t)a.ke[page * a.ke_p + at * a.ke_t + c * a.ke_h] << 23);
          vs8[p] = __uint_as_float((uint32_t)a.ve[page * a.ve_p + at * a.ve_t + c * a.ve_h] << 23);
        }
      }
    }
  };
  auto land = [&](int stage) __attribute__((always_inline)) {   // e4m3: the loads of issue() into LDS
    if constexpr (E4M3) {
      char* dst = smem + stage * 2 * kTileBytes;
#pragma unroll
      for (int p = 0; p < kLoads; ++p) {
        const int i = p * 256 + tid, rr = i / (D / 16), chunk = i % (D / 16);
        bf16x8 lo, hi;
        widen(k8[p], ks8[p], lo, hi);
        *reinterpret_cast<bf16x8*>(dst + L::off(rr, 2 * chunk)) = lo;
        *reinterpret_cast<bf16x8*>(dst + L::off(rr, 2 * chunk + 1)) = hi;
        widen(v8[p], vs8[p], lo, hi);
        *reinterpret_cast<bf16x8*>(dst + kTileBytes + L::off(rr, 2 * chunk)) = lo;
        *reinterpret_cast<bf16x8*>(dst + kTileBytes + L::off(rr, 2 * chunk + 1)) = hi;
      }
    }
  };

  L lo;
  lo.init(lane);
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m_run = first_max(c2), l_run = 0.f;

  // e4m3: a tile is on its way to registers for a whole turn, and goes from there to LDS at the start of the next one
  CacheRow next = look_up(n0);
  uint64_t seen = 0, seen_1 = 0, seen_2 = 0;   // of tiles n, n + 1, n + 2
  if (n0 < n1) {
    seen_1 = seen_of(next);
    issue(next, 0);
    land(0);
    next = look_up(n0 + 1);
    if constexpr (E4M3) {
      seen_2 = seen_of(next);
      issue(next, 1);
      next = look_up(n0 + 2);
    }
  }
  for (int n = n0; n < n1; ++n) {
    const int stage = (n - n0) & 1;
    if constexpr (!E4M3) wait_vmcnt0();   // this wave's part of tile n has landed
    __syncthreads();                      // everyone's part has landed; everyone left tile n - 1
    seen = seen_1;
    if constexpr (E4M3) {
      seen_1 = seen_2;
      if (n + 1 < n1) land(stage ^ 1);
      if (n + 2 < n1) {
        seen_2 = seen_of(next);
        issue(next, stage);
        next = look_up(n + 3);
      }
    } else if (n + 1 < n1) {
      seen_1 = seen_of(next);
      issue(next, stage ^ 1);
      next = look_up(n + 2);
    }
    const int j0 = kt.tile(n) * kKeys;
    const char* Ks = smem + stage * 2 * kTileBytes;
    const char* Vs = Ks + kTileBytes;
    // (bitwise, wave-uniform) nothing of the tile for this wave's rows: after them, or between the sinks and their windows
    const bool skip = idle || j0 > w_hi || (a.window > 0 && j0 + kKeys <= w_lo - a.window + 1 && j0 >= a.sinks);
    if (!skip) {
      f32x16 s0 = zero16(), s1 = zero16();
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        s0 = mfma32(lo.template rm<0>(Ks, k), qf[k], s0);
        s1 = mfma32(lo.template rm<32>(Ks, k), qf[k], s1);
      }
      const bool windowed = a.window > 0 && j0 < w_hi - a.window + 1;
      if (j0 + kKeys - 1 > w_lo || ~seen != 0 || windowed) {
        mask_paged(s0, s1, j0 + 4 * g32, pos, windowed ? p_first + tq - a.window + 1 : 0, a.sinks, seen >> (4 * g32));
      }
      // online softmax: the maximum is raised (and O rescaled) only when it grows by more than 2^8
      float ma = fmaxf(s0[0], s0[1]), mb = fmaxf(s1[0], s1[1]);
#pragma unroll
      for (int v = 2; v < 16; v += 2) {
        ma = fmaxf(fmaxf(ma, s0[v]), s0[v + 1]);
        mb = fmaxf(fmaxf(mb, s1[v]), s1[v + 1]);
      }
      const float mx = max_halves(fmaxf(ma, mb));
      if (__builtin_amdgcn_ballot_w64(mx * c2 > m_run * c2 + 8.f) != 0) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c2);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
      }
      const float mc = m_run * c2;
      float ra = 0.f, rb = 0.f;
      bf16x8 pf[4];
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s0[v] = __builtin_amdgcn_exp2f(fmaf(s0[v], c2, -mc));
        s1[v] = __builtin_amdgcn_exp2f(fmaf(s1[v], c2, -mc));
        ra += s0[v];
        rb += s1[v];
      }
      l_run += ra + rb;
      pf[0] = pack8(s0[0], s0[1], s0[2], s0[3], s0[4], s0[5], s0[6], s0[7]);
      pf[1] = pack8(s0[8], s0[9], s0[10], s0[11], s0[12], s0[13], s0[14], s0[15]);
      pf[2] = pack8(s1[0], s1[1], s1[2], s1[3], s1[4], s1[5], s1[6], s1[7]);
      pf[3] = pack8(s1[8], s1[9], s1[10], s1[11], s1[12], s1[13], s1[14], s1[15]);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        o[db] = mfma32(lo.template tr<0>(Vs, db), pf[0], o[db]);
        o[db] = mfma32(lo.template tr<16>(Vs, db), pf[1], o[db]);
        o[db] = mfma32(lo.template tr<32>(Vs, db), pf[2], o[db]);
        o[db] = mfma32(lo.template tr<48>(Vs, db), pf[3], o[db]);
      }
    }
  }
  __syncthreads();

  if (idle) return;
  chunk_epilogue<D>(a, o, m_run * c2, l_run, smem + w * 32 * L::kRow, sr.s0, c, iw, n_rows, t, h, split, piece.count, lane);
}

// The same for 256 rows: eight waves and three stages, the walk of the eight-wave forward (D = 128).
template <bool E4M3>
__global__ void __launch_bounds__(512, 1) paged_long_kernel(PArgs a, int first_block) {
  constexpr int D = 128, kLog2 = 8, kRows8 = 1 << kLog2, kEsz = E4M3 ? 1 : 2, kStageBytes = 2 * kTileBytes;
  __shared__ __attribute__((aligned(1024))) char smem[3 * kStageBytes];   // [stage][K, V]
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  int tile, c, split;
  if (!tile_of_block(a, a.chunk, first_block + block_id(), tile, c, split)) return;
  const int b = find_seq<kLog2>(a, tile, lane);
  if (b < 0) return;
  const SeqRows sr = seq_rows(a, b);
  const int i0 = uni((tile - first_tile<kLog2>(a, b)) * kRows8), n_rows = uni(sr.n * a.r);
  if (i0 >= n_rows || n_rows <= a.few_rows) return;
  const int p_first = uni(sr.kv - sr.n);
  const int p_lo = uni(p_first + quot(i0, a.by_r));
  const int p_hi = uni(p_first + quot(min(i0 + kRows8, n_rows) - 1, a.by_r));
  const KeyTiles kt = key_tiles<kKeys>(a.window, a.sinks, p_lo, p_hi, sr.keys);
  const Piece piece = pieces_of(a.chunk, kt.total);
  const int n0 = split * piece.per, nt = uni(min(kt.total, n0 + piece.per) - n0);
  if (split > 0 && nt <= 0) return;

  const int iw = i0 + 32 * w, row = min(iw + l32, n_rows - 1);
  const int tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
  const int t = sr.s0 + tq, pos = min(p_first + tq, sr.keys - 1), p_row = p_first + tq;
  const int w_lo = uni(p_first + quot(min(iw, n_rows - 1), a.by_r));
  const int w_hi = uni(p_first + quot(min(iw + 32, n_rows) - 1, a.by_r));
  const bool idle = iw >= n_rows;
  const float c2 = a.scale_log2;
  bf16x8 qf[8];
  {
    const bf16x8* src = reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + t * a.q_t + h * a.q_h);
#pragma unroll
    for (int k = 0; k < 8; ++k) qf[k] = src[2 * k + g32];
  }
  const char* k_head = a.kc + c * a.kc_h * kEsz;
  const char* v_head = a.vc + c * a.vc_h * kEsz;
  const uint32_t smem_base = lds_addr(smem);
  auto look_up = [&](int n) __attribute__((always_inline)) {
    return n < nt ? cache_row(a, b, kt.tile(n0 + n) * kKeys + lane, kt.end) : CacheRow{-1, 0};
  };
  CacheRow next = look_up(0);
  uint64_t seen_a = 0, seen_b = 0;   // of the last two tiles issued
  uint4 k8, v8;                      // e4m3: the tile on its way to LDS
  float ks8, vs8;
  auto issue = [&](int n, int stage) __attribute__((always_inline)) {
    const CacheRow x = next;
    seen_a = seen_b;
    seen_b = __builtin_amdgcn_ballot_w64(x.page >= 0);
    next = look_up(n + 1);
    if constexpr (!E4M3) {
      const uint32_t dst = smem_base + stage * kStageBytes;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int rr = 32 * p + 4 * w + (lane >> 4), chunk = (lane & 15) ^ swz(rr);
        const int page = __shfl(x.page, rr), at = __shfl(x.at, rr);
        const char* zero = reinterpret_cast<const char*>(zero_row);
        const char* ks = page < 0 ? zero : k_head + (page * a.kc_p + at * a.kc_t) * 2;
        const char* vs = page < 0 ? zero : v_head + (page * a.vc_p + at * a.vc_t) * 2;
        dma16(ks + chunk * 16, dst + (32 * p + 4 * w) * kRowBytes);
        dma16(vs + chunk * 16, dst + (32 * p + 4 * w) * kRowBytes + kTileBytes);
      }
    } else {
      const int rr = tid >> 3, chunk = tid & 7;
      const int page = __shfl(x.page, rr), at = __shfl(x.at, rr);
      const char* zero = reinterpret_cast<const char*>(zero_row);
      const bool there = page >= 0;
      k8 = *reinterpret_cast<const uint4*>((there ? k_head + page * a.kc_p + at * a.kc_t : zero) + chunk * 16);
      v8 = *reinterpret_cast<const uint4*>((there ? v_head + page * a.vc_p + at * a.vc_t : zero) + chunk * 16);
      const uint8_t* ze = reinterpret_cast<const uint8_t*>(zero);
      ks8 = __uint_as_float((uint32_t)*(there ? a.ke + page * a.ke_p + at * a.ke_t + c * a.ke_h : ze) << 23);
      vs8 = __uint_as_float((uint32_t)*(there ? a.ve + page * a.ve_p + at * a.ve_t + c * a.ve_h : ze) << 23);
    }
  };
  auto land = [&](int n) __attribute__((always_inline)) {
    if constexpr (E4M3) {
      const int rr = tid >> 3, chunk = tid & 7;
      char* dst = smem + n % 3 * kStageBytes;
      bf16x8 lo, hi;
      widen(k8, ks8, lo, hi);
      *reinterpret_cast<bf16x8*>(dst + tile_off(rr, 2 * chunk)) = lo;
      *reinterpret_cast<bf16x8*>(dst + tile_off(rr, 2 * chunk + 1)) = hi;
      widen(v8, vs8, lo, hi);
      *reinterpret_cast<bf16x8*>(dst + kTileBytes + tile_off(rr, 2 * chunk)) = lo;
      *reinterpret_cast<bf16x8*>(dst + kTileBytes + tile_off(rr, 2 * chunk + 1)) = hi;
    }
  };
  LaneOffsets lo;
  init_lane_offsets(lo, lane);
  FwdState st;
  st.m_run = first_max(c2);
  st.l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) st.o_acc[db] = zero16();
  pp_walk(st, qf, lo, smem, nt, w >> 2, c2, issue, land,
          [&](int n) {
            const int j0 = kt.tile(n0 + n) * kKeys;
            return !idle && j0 <= w_hi && (a.window == 0 || j0 + kKeys > w_lo - a.window + 1 || j0 < a.sinks);
          },
          [&](f32x16& s0, f32x16& s1, int n) {
            const int j0 = kt.tile(n0 + n) * kKeys;
            const uint64_t seen = n + 1 < nt ? seen_a : seen_b;   // the tile after it is on its way already
            const bool windowed = a.window > 0 && j0 < w_hi - a.window + 1;
            if (j0 + kKeys - 1 > w_lo || ~seen != 0 || windowed)
              mask_paged(s0, s1, j0 + 4 * g32, pos, windowed ? p_row - a.window + 1 : 0, a.sinks, seen >> (4 * g32));
          });
  __syncthreads();
  if (idle) return;
  chunk_epilogue<D>(a, st.o_acc, st.m_run * c2, st.l_run, smem + w * 32 * kRowBytes, sr.s0, c, iw, n_rows, t, h, split, piece.count, lane);
}

// ---- few rows.  v_mfma_f32_16x16x32_bf16, lane l: c16 = l % 16, q4 = l / 16 (operand layout: s2attn_bf16_common.h).
// K and V of a 32-key tile take the same way to registers: lane (c16, q4) has of the keys c16 and c16 + 16 every fourth 16-byte
// piece from the q4-th on, so it looks up two keys and no lane needs another's.  K is the A operand as it comes (which d
// a contraction slot stands for is free as long as Q agrees: with e4m3 a piece is 16 values, two operands); V goes through the
// wave's own part of LDS, which turns it.
template <int D, bool E4M3>
struct FewTile {
  static constexpr int N = D / (E4M3 ? 64 : 32);   // pieces of a key and lane
  uint4 k[2][N], v[2][N];
  float ks[2], vs[2];                              // e4m3: scales
  uint32_t seen;                                   // a bit for each key that exists
};

template <int D, bool E4M3, int NQ>
__device__ __forceinline__ void few_workgroup(const PArgs& a, int block, char* smem) {
  using T = FewTile<D, E4M3>;
  constexpr int TK = 32, kWaves = 4, kRow = D * 2, KF = D / 32, DB = D / 16;   // KF: operands of a key over D
  constexpr int kEsz = E4M3 ? 1 : 2, kStride = D + 4;                          // kStride: floats of a row of the sums
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int c16 = lane & 15, q4 = lane >> 4;
  const int y = quot(block, a.by_Hkv), c = block - y * a.Hkv;
  const int b = quot(y, a.few.by_splits), split = y - b * a.few.splits;
  if (b >= a.B) return;
  const SeqRows sr = seq_rows(a, b);
  const int n_rows = uni(sr.n * a.r), p_first = uni(sr.kv - sr.n);
  if (n_rows > a.few_rows) return;

  const char* k_head = a.kc + c * a.kc_h * kEsz + 16 * q4;
  const char* v_head = a.vc + c * a.vc_h * kEsz + 16 * q4;
  float* blocks = reinterpret_cast<float*>(smem);
  float* max_s = blocks + kWaves * 16 * NQ * kStride;                          // [wave][row]
  float* sum_s = max_s + kWaves * 16 * NQ;
  char* Vs = smem + w * (TK * kRow);

  // transposed operand of V: rows 4 q4 + c16 / 4 (and 16 further) of columns 16 db + 4 (c16 % 4) ..
  int tr[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int row = 4 * q4 + (c16 >> 2), col = 16 * db + 4 * (c16 & 3);
    tr[db] = Tile<D>::off(row, col >> 3) + (col & 7) * 2;
  }

  for (int i0 = 0; i0 < n_rows; i0 += 16 * NQ) {
    const int p_lo = uni(p_first + quot(i0, a.by_r)), p_hi = uni(p_first + quot(min(i0 + 16 * NQ, n_rows) - 1, a.by_r));
    const KeyTiles kt = key_tiles<TK>(a.window, a.sinks, p_lo, p_hi, sr.keys);
    const Piece piece = pieces_of(a.few, kt.total);
    const int per = piece.per, n0 = split * per, n1 = uni(min(kt.total, n0 + per));
    if (split > 0 && n0 >= n1) continue;

    auto look_up = [&](int n, CacheRow (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) x[kb] = n < n1 ? cache_row(a, b, kt.tile(n) * TK + 16 * kb + c16, kt.end) : CacheRow{-1, 0};
    };
    auto load = [&](T& t, const CacheRow (&x)[2]) __attribute__((always_inline)) {
      t.seen = ((uint32_t)__builtin_amdgcn_ballot_w64(x[0].page >= 0) & 0xffffu) |
               ((uint32_t)__builtin_amdgcn_ballot_w64(x[1].page >= 0) << 16);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bool there = x[kb].page >= 0;
        const char* zero = reinterpret_cast<const char*>(zero_row);
        const char* kp = there ? k_head + (x[kb].page * a.kc_p + x[kb].at * a.kc_t) * kEsz : zero;
        const char* vp = there ? v_head + (x[kb].page * a.vc_p + x[kb].at * a.vc_t) * kEsz : zero;
#pragma unroll
        for (int i = 0; i < T::N; ++i) t.k[kb][i] = *reinterpret_cast<const uint4*>(kp + 64 * i);
#pragma unroll
        for (int i = 0; i < T::N; ++i) t.v[kb][i] = *reinterpret_cast<const uint4*>(vp + 64 * i);
        if constexpr (E4M3) {
          const uint8_t* ke = there ? a.ke + x[kb].page * a.ke_p + x[kb].at * a.ke_t + c * a.ke_h : reinterpret_cast<const uint8_t*>(zero);
          const uint8_t* ve = there ? a.ve + x[kb].page * a.ve_p + x[kb].at * a.ve_t + c * a.ve_h : reinterpret_cast<const uint8_t*>(zero);
          t.ks[kb] = __uint_as_float((uint32_t)*ke << 23);
          t.vs[kb] = __uint_as_float((uint32_t)*ve << 23);
        }
      }
    };

    // this wave's tiles: n0 + w, n0 + w + 4, ..
    // The look-up of a tile goes out ahead of the loads of the tile before it, so that waiting for it is not waiting for them.
    T ta, tb;
    CacheRow at[2], at_next[2];
    look_up(n0 + w, at);
    look_up(n0 + w + kWaves, at_next);
    load(ta, at);

    bf16x8 qf[NQ][KF];
    int pos[NQ], p_row[NQ];
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const int row = min(i0 + 16 * qb + c16, n_rows - 1), tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
      p_row[qb] = p_first + tq;
      pos[qb] = min(p_row[qb], sr.keys - 1);
      const __bf16* q = static_cast<const __bf16*>(a.q) + (sr.s0 + tq) * a.q_t + h * a.q_h;
#pragma unroll
      for (int f = 0; f < KF; ++f)
        qf[qb][f] = *reinterpret_cast<const bf16x8*>(q + (E4M3 ? 16 * (q4 + 4 * (f >> 1)) + 8 * (f & 1) : 32 * f + 8 * q4));
    }
    f32x4 o[DB][NQ];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) o[db][qb] = zero4();
    float m_run[NQ], l_run[NQ];   // base 2; finite: weights of zero, not NaN, where no key so far is visible
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) { m_run[qb] = -3.402823466e38f; l_run[qb] = 0.f; }
    const float c2 = a.scale_log2;

    auto step = [&](T& cur, T& nxt, int n) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) at[kb] = at_next[kb];
      look_up(n + 2 * kWaves, at_next);
      if constexpr (NQ == 1) load(nxt, at);   // (past the end: zeros)
      const int j0 = kt.tile(n) * TK;
      const uint32_t seen = cur.seen;
      // V into LDS, K as operands
      f32x4 sc[2][NQ];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        bf16x8 kf[KF];
        if constexpr (E4M3) {
#pragma unroll
          for (int i = 0; i < T::N; ++i) {
            bf16x8 x, y2;
            widen(cur.v[kb][i], cur.vs[kb], x, y2);
            *reinterpret_cast<bf16x8*>(Vs + Tile<D>::off(16 * kb + c16, 2 * (q4 + 4 * i))) = x;
            *reinterpret_cast<bf16x8*>(Vs + Tile<D>::off(16 * kb + c16, 2 * (q4 + 4 * i) + 1)) = y2;
            widen(cur.k[kb][i], cur.ks[kb], kf[2 * i], kf[2 * i + 1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < T::N; ++i) {
            *reinterpret_cast<uint4*>(Vs + Tile<D>::off(16 * kb + c16, q4 + 4 * i)) = cur.v[kb][i];
            kf[i] = __builtin_bit_cast(bf16x8, cur.k[kb][i]);
          }
        }
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          sc[kb][qb] = zero4();
#pragma unroll
          for (int f = 0; f < KF; ++f) sc[kb][qb] = mfma16(kf[f], qf[qb][f], sc[kb][qb]);
        }
      }
      wave_lds_order();
      if constexpr (NQ > 1) load(nxt, at);
      const bool windowed = a.window > 0 && j0 < p_hi - a.window + 1;
      const bool masked = j0 + TK - 1 > p_lo || ~seen != 0 || windowed;
      const uint32_t seen_l = seen >> (4 * q4);
      bf16x8 pf[NQ];
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        const int first = windowed ? p_row[qb] - a.window + 1 : 0;
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = sc[kb][qb][e] * c2;
            const int key = j0 + 16 * kb + 4 * q4 + e;
            if (masked && !(key <= pos[qb] && (key >= first || key < a.sinks) && (seen_l >> (16 * kb + e) & 1))) x = -INFINITY;
            sc[kb][qb][e] = x;
            mx = fmaxf(mx, x);
          }
        mx = max_of_4(mx);
        if (__builtin_amdgcn_ballot_w64(mx > m_run[qb]) != 0) {
          const float m_new = fmaxf(m_run[qb], mx);
          const float alpha = __builtin_amdgcn_exp2f(m_run[qb] - m_new);
          m_run[qb] = m_new;
          l_run[qb] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db][qb] *= alpha;
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[kb][qb][e] = __builtin_amdgcn_exp2f(sc[kb][qb][e] - m_run[qb]);
            l_run[qb] += sc[kb][qb][e];
          }
        pf[qb] = pack8(sc[0][qb], sc[1][qb]);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(S2_LDS(bf16x4, Vs + tr[db]));
        const bf16x4 y2 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(S2_LDS(bf16x4, Vs + tr[db] + 16 * kRow));
        const bf16x8 vf = __builtin_shufflevector(x, y2, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) o[db][qb] = mfma16(vf, pf[qb], o[db][qb]);
      }
      wave_lds_order();
    };
    if constexpr (NQ == 1) {
      for (int n = n0 + w; n < n1; n += 2 * kWaves) {
        step(ta, tb, n);
        if (n + kWaves < n1) step(tb, ta, n + kWaves);
      }
    } else {   // two row blocks leave no registers for a second tile: the next one is asked for as soon as this one is in use
      for (int n = n0 + w; n < n1; n += kWaves) step(ta, ta, n);
    }

    // ---- the waves' sums meet
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) l_run[qb] = sum_of_4(l_run[qb]);
    __syncthreads();   // every wave is done with its V
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<f32x4*>(blocks + (w * 16 * NQ + 16 * qb + c16) * kStride + 16 * db + 4 * q4) = o[db][qb];
      if (q4 == 0) {
        max_s[w * 16 * NQ + 16 * qb + c16] = m_run[qb];
        sum_s[w * 16 * NQ + 16 * qb + c16] = l_run[qb];
      }
    }
    __syncthreads();
    constexpr int kLanes = D / 8, kAtOnce = 256 / kLanes;   // rows at once: 16 or 32
#pragma unroll
    for (int pass = 0; pass < (16 * NQ + kAtOnce - 1) / kAtOnce; ++pass) {
      const int row = pass * kAtOnce + tid / kLanes, ch = tid % kLanes;
      if (row >= 16 * NQ || i0 + row >= n_rows) continue;
      float m = max_s[row], l = 0.f;
#pragma unroll
      for (int x = 1; x < kWaves; ++x) m = fmaxf(m, max_s[x * 16 * NQ + row]);
      f32x4 s0 = zero4(), s1 = zero4();
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float f = __builtin_amdgcn_exp2f(max_s[x * 16 * NQ + row] - m);
        l = fmaf(sum_s[x * 16 * NQ + row], f, l);
        const f32x4* p = reinterpret_cast<const f32x4*>(blocks + (x * 16 * NQ + row) * kStride + 8 * ch);
        s0 += p[0] * f;
        s1 += p[1] * f;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
      const int tq = quot(i0 + row, a.by_r), h = c * a.r + i0 + row - tq * a.r, t = sr.s0 + tq, H = a.Hkv * a.r;
      if (piece.count > 1) {
        const size_t dst = ((size_t)split * a.T + t) * H + h;
        f32x4* po = reinterpret_cast<f32x4*>(a.part_o + dst * D + 8 * ch);
        po[0] = s0 * inv;
        po[1] = s1 * inv;
        if (ch == 0) a.part_lse[dst] = lse2;
      } else {
        *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(a.o) + ((size_t)t * H + h) * D + 8 * ch) = pack8(s0 * inv, s1 * inv);
        if (ch == 0 && a.lse) a.lse[(size_t)h * a.T + t] = lse2 * kLn2;
      }
    }
    __syncthreads();   // before the next rows' V
  }
}

template <int D>
constexpr int kChunkBytes = 4 * kKeys * Tile<D>::kRow;
template <int D, int NQ>
constexpr int kFewBytes = 4 * 16 * NQ * (D + 4 + 2) * 4 > 4 * 32 * D * 2 ? 4 * 16 * NQ * (D + 4 + 2) * 4 : 4 * 32 * D * 2;

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_chunk_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kChunkBytes<D>];
  chunk_workgroup<D, E4M3>(a, first_block + block_id(), smem);
}

template <int D, bool E4M3, int NQ>
__global__ void __launch_bounds__(256, 2) paged_few_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kFewBytes<D, NQ>];
  few_workgroup<D, E4M3, NQ>(a, first_block + block_id(), smem);
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_both_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kChunkBytes<D> > kFewBytes<D, 2> ? kChunkBytes<D> : kFewBytes<D, 2>];
  const int block = first_block + block_id();
  if (block < a.chunk_blocks)
    chunk_workgroup<D, E4M3>(a, block, smem);
  else
    few_workgroup<D, E4M3, 2>(a, block - a.chunk_blocks, smem);
}

template <int D, bool E4M3>
int launch_t(const PArgs& a, int nq, hipStream_t st) {
  const int few = a.B * a.Hkv * a.few.splits;
  if constexpr (D == 128) {
    if (a.chunk_blocks > 0 && a.chunk_rows == 256) {
      const int rc = launch_blocks(paged_long_kernel<E4M3>, a.chunk_blocks, 512, st, a);
      return rc != 0 || a.few_rows == 0 ? rc : launch_blocks(paged_few_kernel<D, E4M3, 2>, few, 256, st, a);
    }
  }
  if (a.few_rows == 0) return launch_blocks(paged_chunk_kernel<D, E4M3>, a.chunk_blocks, 256, st, a);
  if (a.chunk_blocks > 0) return launch_blocks(paged_both_kernel<D, E4M3>, a.chunk_blocks + few, 256, st, a);
  return nq == 1 ? launch_blocks(paged_few_kernel<D, E4M3, 1>, few, 256, st, a) : launch_blocks(paged_few_kernel<D, E4M3, 2>, few, 256, st, a);
}

}  // namespace

int launch_paged_bf16(const PArgs& a, int D, bool e4m3, int nq, hipStream_t st) {
  if (D == 64) return e4m3 ? launch_t<64, true>(a, nq, st) : launch_t<64, false>(a, nq, st);
  return e4m3 ? launch_t<128, true>(a, nq, st) : launch_t<128, false>(a, nq, st);
}

}  // namespace s2
