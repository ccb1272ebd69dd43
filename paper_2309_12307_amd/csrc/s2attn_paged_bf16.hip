// bf16 attention of new tokens over a paged cache (bf16 or e4m3) for gfx950.
//
// The rows of one sequence and kv head are its (token, query head of the kv head) pairs, token by token, so that K and V
// are read once for all query heads that share them.  Two kinds of workgroup (4 waves) share a launch:
//   chunk  128 rows of a sequence that has many, and a piece of their keys; a wave owns 32 rows, the waves share the
//          64-key tiles, staged in LDS.  S^T = K Q^T, online softmax, O^T += V^T P^T as in the forward kernels on contiguous
//          tensors.  Bound by the matrix unit (2048 rows over 32768 keys, H = 32, D = 128: 990 us, 1080 TFLOP/s; D = 64 by the vector
//          unit, which has twice the exponentials for a product).
//   few    all rows of a sequence that has up to 16 (e4m3: 32), as single tokens have, or as many of its tokens as make that, and a
//          piece of its keys; the waves take different 32-key tiles and meet once, at the end.  Bound by HBM: what counts is bytes
//          on the way, so a wave has a whole tile of K and V on its way to registers while it works on another, and waits for
//          nobody (two sequences over 100 000 tokens, e4m3, 32 kv heads: 290 us, 5.7 TB/s; 32 over up to 8192, bf16, 8 kv heads: 86
//          us and the join 5).
// Rows that several pieces share leave normalised fp32 partial outputs and their log-sum-exp, which a second kernel joins.
//
// P is rounded to bf16 for the second product (as everywhere in this library); the row sum adds the unrounded P, and
// statistics, outputs and partial outputs stay fp32 up to the one rounding of o.
#include <type_traits>

#include "s2attn_bf16_fwd.h"
#include "s2attn_bf16_tile.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

constexpr int kKeys = 64;       // of a tile
constexpr int kRowsLog2 = 7;
constexpr int kRows = 1 << kRowsLog2;

// Removes the scores of keys that this lane's row does not see: those but the `n` up to `pos` and the sinks up to it, and those on
// pages that do not exist.  `key0`: this lane's first key; `seen`: a bit a key from there on.
__device__ __forceinline__ void mask_paged(f32x16& s0, f32x16& s1, int key0, int pos, int n, int sinks, uint64_t seen) {
  int d0 = pos - key0;
  asm volatile("" : "+v"(d0));   // keeps the compiler from doing all this ahead of the branch that asks for it
  const int last = min(pos, sinks - 1) - key0;   // keys up to it are sinks that the row sees
  const uint32_t seen0 = (uint32_t)seen, seen1 = (uint32_t)(seen >> 32);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int bit = 8 * (v >> 2) + (v & 3);
    s0[v] = ((((unsigned)(d0 - bit) < (unsigned)n) | (bit <= last)) & (seen0 >> bit & 1)) ? s0[v] : -INFINITY;
    s1[v] = ((((unsigned)(d0 - bit - 32) < (unsigned)n) | (bit + 32 <= last)) & (seen1 >> bit & 1)) ? s1[v] : -INFINITY;
  }
}

// A wave's 32 rows from iw on (lane l and l + 32: row l, token t and head h): o / l and the log-sum-exp, as a piece or as the
// output, the latter turned through the wave's part of LDS.  A row that saw nothing: 0 and -infinity.  m2: maximum, base 2.
template <int D>
__device__ __forceinline__ void chunk_epilogue(const f32x16 (&o)[D / 32], float m2, float l_run, char* region, int s0, int c,
                                               int iw, int n_rows, int t, int h, int split, int pieces, int lane) {
  using L = Tile<D>;
  constexpr int DB = D / 32, kChunks = D / 8, kRowsPer = 64 / kChunks;
  const PArgs a = late_args();
  const int g32 = lane >> 5, l32 = lane & 31;
  const float l_tot = sum_halves(l_run);
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  const float lse2 = l_tot == 0.f ? -INFINITY : m2 + __builtin_amdgcn_logf(l_tot);
  const bool valid = iw + l32 < n_rows;
  const int H = a.Hkv * a.r;
  if (pieces > 1) {
    if (!valid) return;
    const size_t at = part_row(a, a.chunk, false, split, 0, c, 0, t, h);
    float* dst = a.chunk.part_o + at * D + 4 * g32;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int vv = 0; vv < 4; ++vv)
        *reinterpret_cast<float4*>(dst + 32 * db + 8 * vv) =
            make_float4(o[db][4 * vv] * inv, o[db][4 * vv + 1] * inv, o[db][4 * vv + 2] * inv, o[db][4 * vv + 3] * inv);
    if (g32 == 0) a.chunk.part_lse[at] = lse2;
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
template <int D, bool E4M3, bool BY16>
__device__ __forceinline__ void chunk_workgroup(const PArgs& a, int block, char* smem, int* flags) {
  using L = Tile<D>;
  constexpr int kTileBytes = kKeys * L::kRow;
  constexpr int KS = D / 16, DB = D / 32, kChunks = D / 8;      // k-steps, column blocks, 16-byte chunks of a bf16 row
  constexpr int kEsz = E4M3 ? 1 : 2;
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  int tile, c, split;
  if (!tile_of_block(a, a.chunk, block, tile, c, split)) return;
  const SeqRows sr = find_rows<kRowsLog2>(a, tile, lane);
  const int b = sr.b;
  if (b < 0) return;
  const int i0 = uni((tile - first_tile<kRowsLog2>(a, sr.s0, b)) * kRows), n_rows = uni(sr.n * a.r);
  if (i0 < 0 || i0 >= n_rows || n_rows <= a.few_rows) return;   // (less than 0: row_start falls somewhere)
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
  const int t = sr.s0 + tq, pos = min(p_first + tq, sr.keys - 1), n_seen = keys_up_to(a.window, p_first + tq, pos);
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

  const uint64_t k_head = reinterpret_cast<uint64_t>(a.kc) + c * a.kc_h * kEsz;
  const uint64_t v_head = reinterpret_cast<uint64_t>(a.vc) + c * a.vc_h * kEsz;
  const uint64_t ke_head = reinterpret_cast<uint64_t>(a.ke) + c * a.ke_h, ve_head = reinterpret_cast<uint64_t>(a.ve) + c * a.ve_h;
  const uint32_t smem_base = lds_addr(smem);
  // Every wave looks up all 64 keys of a tile, one a lane, or the four groups of 16 of it; wave w stages the w-th 16 rows.
  // bf16: global -> LDS, a lane's 16 bytes where the layout has the chunk; rows that are not there are zeros.  e4m3: through
  // registers, 16 values to two chunks.
  constexpr int kLine = E4M3 ? D / 16 : kChunks;                // 16-byte pieces of a cached row
  constexpr int kRowsPer = 64 / kLine, kPass = 16 / kRowsPer;   // rows of a wave's load, and its loads
  const int sub = lane / kLine;                                 // this lane's row of the first load
  auto chunk_of = [&](int p) __attribute__((always_inline)) {   // its piece of the row (16 w rows further the layout is the same)
    return E4M3 ? lane % kLine : D == 128 ? (lane & 15) ^ (sub << 2) ^ p : (lane & 7) ^ swz64((p * kRowsPer + sub) >> 1);
  };
  const uint32_t k_sub = (uint32_t)(sub * (int)a.kc_t * kEsz), v_sub = (uint32_t)(sub * (int)a.vc_t * kEsz);
  struct Ahead {   // what is known of a tile before its loads go out: this lane's key, or the page of this wave's group
    CacheRow row;
    int page;
  };
  Plain plain{};
  if constexpr (BY16) plain = plain_tiles<kKeys, 256>(a, b, kt, n0, n1, tid, flags);
  auto look_up = [&](int n) __attribute__((always_inline)) {
    Ahead x;
    if constexpr (BY16) x.page = groups_of<1>(a, b, kt.tile(min(n, n1 - 1)) * kKeys + 16 * w).page[0];
    else x.row = cache_row(a, b, kt.tile(n) * kKeys + lane, n < n1 && is_seen(a, p_lo, kt.end, kt.tile(n) * kKeys + lane));
    return x;
  };
  u32x4 k8[2][kPass], v8[2][kPass];                             // e4m3: two tiles on their way
  float ks8[2][kPass], vs8[2][kPass];
  // Starts the loads of tile n; a bit for each key that exists and that some row sees.
  auto issue = [&](const Ahead& x, int n, int stage) __attribute__((always_inline)) {
    const uint32_t dst = smem_base + stage * 2 * kTileBytes + w * kPass * 1024;
    const uint64_t zero = zero_address();
    if constexpr (BY16) {
      const int j0 = kt.tile(min(n, n1 - 1)) * kKeys, at = place_of(a, j0 + 16 * w);
      const uint64_t kb = k_head + group_off(x.page, at, a.kc_p * kEsz, a.kc_t * kEsz);
      const uint64_t vb = v_head + group_off(x.page, at, a.vc_p * kEsz, a.vc_t * kEsz);
      uint64_t seen = ~0ull;
      const bool all = n >= plain.from && n < plain.to;
      if (!all) seen = n < n1 ? seen_of<4>(a, groups_of<4>(a, b, j0), p_lo, kt.end, j0) : 0;
      const uint32_t mine = (uint32_t)(seen >> (16 * w)) & 0xffffu;
#pragma unroll
      for (int p = 0; p < kPass; ++p) {
        const uint64_t kp = kb + p * kRowsPer * (uint32_t)(a.kc_t * kEsz);
        const uint64_t vp = vb + p * kRowsPer * (uint32_t)(a.vc_t * kEsz);
        const int rr = p * kRowsPer + sub, ch = chunk_of(p) * 16;
        if constexpr (!E4M3) {
          if (all) {
            dma16s(uni64(kp), k_sub + ch, dst + p * 1024);
            dma16s(uni64(vp), v_sub + ch, dst + p * 1024 + kTileBytes);
          } else {
            const bool there = mine >> rr & 1;
            dma16(reinterpret_cast<const void*>((there ? kp + k_sub : zero) + ch), dst + p * 1024);
            dma16(reinterpret_cast<const void*>((there ? vp + v_sub : zero) + ch), dst + p * 1024 + kTileBytes);
          }
        } else {
          const uint64_t ke = ke_head + x.page * a.ke_p + at * a.ke_t;
          const uint64_t ve = ve_head + x.page * a.ve_p + at * a.ve_t;
          const bool there = mine >> rr & 1;
          k8[stage][p] = load16((there ? kp + k_sub : zero) + ch);
          v8[stage][p] = load16((there ? vp + v_sub : zero) + ch);
          ks8[stage][p] = load_scale(there ? ke + (uint32_t)(rr * (int)a.ke_t) : zero);
          vs8[stage][p] = load_scale(there ? ve + (uint32_t)(rr * (int)a.ve_t) : zero);
        }
      }
      return seen;
    } else {
      const CacheRow r = x.row;
#pragma unroll
      for (int p = 0; p < kPass; ++p) {
        const int rr = 16 * w + p * kRowsPer + sub, ch = chunk_of(p) * 16;
        const int page = __shfl(r.page, rr), at = __shfl(r.at, rr);
        const bool there = page >= 0;
        const uint64_t ks = (there ? k_head + (page * a.kc_p + at * a.kc_t) * kEsz : zero) + ch;
        const uint64_t vs = (there ? v_head + (page * a.vc_p + at * a.vc_t) * kEsz : zero) + ch;
        if constexpr (!E4M3) {
          dma16(reinterpret_cast<const void*>(ks), dst + p * 1024);
          dma16(reinterpret_cast<const void*>(vs), dst + p * 1024 + kTileBytes);
        } else {
          k8[stage][p] = load16(ks);
          v8[stage][p] = load16(vs);
          ks8[stage][p] = load_scale(there ? ke_head + page * a.ke_p + at * a.ke_t : zero);
          vs8[stage][p] = load_scale(there ? ve_head + page * a.ve_p + at * a.ve_t : zero);
        }
      }
      return (uint64_t)__builtin_amdgcn_ballot_w64(r.page >= 0);
    }
  };
  auto land = [&](int stage) __attribute__((always_inline)) {   // e4m3: the loads of issue() into LDS
    if constexpr (E4M3) {
      char* dst = smem + stage * 2 * kTileBytes;
#pragma unroll
      for (int p = 0; p < kPass; ++p) {
        const int rr = 16 * w + p * kRowsPer + sub;
        bf16x8 lo, hi;
        widen(k8[stage][p], ks8[stage][p], lo, hi);
        *reinterpret_cast<bf16x8*>(dst + L::off(rr, 2 * chunk_of(p))) = lo;
        *reinterpret_cast<bf16x8*>(dst + L::off(rr, 2 * chunk_of(p) + 1)) = hi;
        widen(v8[stage][p], vs8[stage][p], lo, hi);
        *reinterpret_cast<bf16x8*>(dst + kTileBytes + L::off(rr, 2 * chunk_of(p))) = lo;
        *reinterpret_cast<bf16x8*>(dst + kTileBytes + L::off(rr, 2 * chunk_of(p) + 1)) = hi;
      }
    }
  };

  L lo;
  lo.init(lane);
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = zero16();
  float m_run = first_max(c2), l_run = 0.f;

  // e4m3: a tile is on its way to registers for two turns, and goes from there to LDS at the start of the turn before its own
  Ahead next{};
  uint64_t seen = 0, seen_1 = 0, seen_2 = 0, seen_3 = 0;   // of tiles n, n + 1, n + 2, n + 3
  if (n0 < n1) {
    next = look_up(n0);
    seen_1 = issue(next, n0, 0);
    next = look_up(n0 + 1);
    if constexpr (E4M3) {
      seen_2 = issue(next, n0 + 1, 1);
      next = look_up(n0 + 2);
      land(0);
      seen_3 = issue(next, n0 + 2, 0);
      next = look_up(n0 + 3);
    }
  }
  auto turn = [&](auto stage_c, int n) __attribute__((always_inline)) {
    constexpr int stage = decltype(stage_c)::value;
    if constexpr (!E4M3) wait_vmcnt0();   // this wave's part of tile n has landed
    __syncthreads();                      // everyone's part has landed; everyone left tile n - 1
    seen = seen_1;
    if constexpr (E4M3) {
      seen_1 = seen_2;
      seen_2 = seen_3;
      land(stage ^ 1);                    // tile n + 1 (past the end: zeros)
      const Ahead x = next;
      next = look_up(n + 4);              // ahead of the loads, so that waiting for it is not waiting for them
      seen_3 = issue(x, n + 3, stage ^ 1);
    } else if (n + 1 < n1) {
      seen_1 = issue(next, n + 1, stage ^ 1);
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
      if (j0 + kKeys - 1 > w_lo || ~seen != 0 || (a.window > 0 && j0 < w_hi - a.window + 1))
        mask_paged(s0, s1, j0 + 4 * g32, pos, n_seen, a.window > 0 ? a.sinks : 0, seen >> (4 * g32));
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
  };
  for (int n = n0; n < n1; n += 2) {
    turn(std::integral_constant<int, 0>{}, n);
    if (n + 1 < n1) turn(std::integral_constant<int, 1>{}, n + 1);
  }
  __syncthreads();

  if (idle) return;
  chunk_epilogue<D>(o, m_run * c2, l_run, smem + w * 32 * L::kRow, sr.s0, c, iw, n_rows, t, h, split, piece.count, lane);
}

// The same for 256 rows: eight waves and three stages, the walk of the eight-wave forward (D = 128, pages of a multiple of 16).
template <bool E4M3>
__global__ void __launch_bounds__(512, 1) paged_long_kernel(PArgs a, int first_block) {
  constexpr int D = 128, kLog2 = 8, kRows8 = 1 << kLog2, kEsz = E4M3 ? 1 : 2, kStageBytes = 2 * kTileBytes;
  __shared__ __attribute__((aligned(1024))) char smem[3 * kStageBytes];   // [stage][K, V]
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  int tile, c, split;
  if (!tile_of_block(a, a.chunk, first_block + block_id(), tile, c, split)) return;
  const SeqRows sr = find_rows<kLog2>(a, tile, lane);
  const int b = sr.b;
  if (b < 0) return;
  const int i0 = uni((tile - first_tile<kLog2>(a, sr.s0, b)) * kRows8), n_rows = uni(sr.n * a.r);
  if (i0 < 0 || i0 >= n_rows || n_rows <= a.few_rows) return;   // (less than 0: row_start falls somewhere)
  const int p_first = uni(sr.kv - sr.n);
  const int p_lo = uni(p_first + quot(i0, a.by_r));
  const int p_hi = uni(p_first + quot(min(i0 + kRows8, n_rows) - 1, a.by_r));
  const KeyTiles kt = key_tiles<kKeys>(a.window, a.sinks, p_lo, p_hi, sr.keys);
  const Piece piece = pieces_of(a.chunk, kt.total);
  const int n0 = split * piece.per, nt = uni(min(kt.total, n0 + piece.per) - n0);
  if (split > 0 && nt <= 0) return;

  const int iw = i0 + 32 * w, row = min(iw + l32, n_rows - 1);
  const int tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
  const int t = sr.s0 + tq, pos = min(p_first + tq, sr.keys - 1), n_seen = keys_up_to(a.window, p_first + tq, pos);
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
  const uint64_t k_head = reinterpret_cast<uint64_t>(a.kc) + c * a.kc_h * kEsz;
  const uint64_t v_head = reinterpret_cast<uint64_t>(a.vc) + c * a.vc_h * kEsz;
  const uint64_t ke_head = reinterpret_cast<uint64_t>(a.ke) + c * a.ke_h, ve_head = reinterpret_cast<uint64_t>(a.ve) + c * a.ve_h;
  const uint32_t smem_base = lds_addr(smem);
  // wave w stages rows 8 w .. 8 w + 7, half a group of 16
  constexpr int kPass = E4M3 ? 1 : 2;
  const int sub = E4M3 ? lane >> 3 : lane >> 4;
  const uint32_t k_sub = (uint32_t)(sub * (int)a.kc_t * kEsz), v_sub = (uint32_t)(sub * (int)a.vc_t * kEsz);
  __shared__ int flags[8];
  const Plain plain = plain_tiles<kKeys, 512>(a, b, kt, n0, n0 + nt, tid, flags);
  auto look_up = [&](int n) __attribute__((always_inline)) {
    return groups_of<1>(a, b, kt.tile(n0 + max(min(n, nt - 1), 0)) * kKeys + 8 * w).page[0];
  };
  int next = look_up(0);
  uint64_t seen_a = 0, seen_b = 0;   // of the last two tiles issued
  u32x4 k8, v8;                      // e4m3: the tile on its way to LDS
  float ks8, vs8;
  auto issue = [&](int n, int stage) __attribute__((always_inline)) {
    const int page = next;
    next = look_up(n + 1);
    const int j0 = kt.tile(n0 + n) * kKeys, at = place_of(a, j0 + 8 * w);
    const bool all = n0 + n >= plain.from && n0 + n < plain.to;
    seen_a = seen_b;
    seen_b = ~0ull;
    if (!all) seen_b = seen_of<4>(a, groups_of<4>(a, b, j0), p_lo, kt.end, j0);
    const uint32_t dst = smem_base + stage * kStageBytes + 8 * w * kRowBytes;
    const uint64_t zero = zero_address();
    const uint64_t kb = k_head + group_off(page, at, a.kc_p * kEsz, a.kc_t * kEsz);
    const uint64_t vb = v_head + group_off(page, at, a.vc_p * kEsz, a.vc_t * kEsz);
    const uint32_t mine = (uint32_t)(seen_b >> (8 * w)) & 0xffu;
#pragma unroll
    for (int p = 0; p < kPass; ++p) {
      const uint64_t kp = kb + 4 * p * (uint32_t)(a.kc_t * kEsz);
      const uint64_t vp = vb + 4 * p * (uint32_t)(a.vc_t * kEsz);
      const int ch = (E4M3 ? lane & 7 : (lane & 15) ^ swz(8 * (w & 1) + 4 * p + sub)) * 16;
      const bool there = mine >> (4 * p + sub) & 1;
      if constexpr (!E4M3) {
        if (all) {
          dma16s(uni64(kp), k_sub + ch, dst + 4 * p * kRowBytes);
          dma16s(uni64(vp), v_sub + ch, dst + 4 * p * kRowBytes + kTileBytes);
        } else {
          dma16(reinterpret_cast<const void*>((there ? kp + k_sub : zero) + ch), dst + 4 * p * kRowBytes);
          dma16(reinterpret_cast<const void*>((there ? vp + v_sub : zero) + ch), dst + 4 * p * kRowBytes + kTileBytes);
        }
      } else {
        const uint64_t ke = ke_head + page * a.ke_p + at * a.ke_t;
        const uint64_t ve = ve_head + page * a.ve_p + at * a.ve_t;
        k8 = load16((there ? kp + k_sub : zero) + ch);
        v8 = load16((there ? vp + v_sub : zero) + ch);
        ks8 = load_scale(there ? ke + (uint32_t)(sub * (int)a.ke_t) : zero);
        vs8 = load_scale(there ? ve + (uint32_t)(sub * (int)a.ve_t) : zero);
      }
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
            if (j0 + kKeys - 1 > w_lo || ~seen != 0 || (a.window > 0 && j0 < w_hi - a.window + 1))
              mask_paged(s0, s1, j0 + 4 * g32, pos, n_seen, a.window > 0 ? a.sinks : 0, seen >> (4 * g32));
          });
  __syncthreads();
  if (idle) return;
  chunk_epilogue<D>(st.o_acc, st.m_run * c2, st.l_run, smem + w * 32 * kRowBytes, sr.s0, c, iw, n_rows, t, h, split, piece.count, lane);
}

// ---- few rows.  v_mfma_f32_16x16x32_bf16, lane l: c16 = l % 16, q4 = l / 16 (operand layout: s2attn_bf16_common.h).
// K and V of a 32-key tile take the same way to registers: lane (c16, q4) has of the keys c16 and c16 + 16 every fourth 16-byte
// piece from the q4-th on, so it looks up two keys and no lane needs another's.  K is the A operand as it comes (which d
// a contraction slot stands for is free as long as Q agrees: with e4m3 a piece is 16 values, two operands); V goes through the
// wave's own part of LDS, which turns it.
template <int D, bool E4M3>
struct FewTile {
  static constexpr int N = D / (E4M3 ? 64 : 32);   // pieces of a key and lane
  u32x4 k[2][N], v[2][N];
  float ks[2], vs[2];                              // e4m3: scales
  uint32_t seen;                                   // a bit for each key that exists and that some row sees
};

// BOTH: beside the other kind of workgroup
template <int D, bool E4M3, bool BY16, int NQ, bool BOTH>
__device__ __forceinline__ void few_workgroup(const PArgs& a, int block, char* smem) {
  using T = FewTile<D, E4M3>;
  constexpr int TK = 32, kWaves = 4, kRow = D * 2, KF = D / 32, DB = D / 16;   // KF: operands of a key over D
  constexpr int kEsz = E4M3 ? 1 : 2, kStride = D + 4;                          // kStride: floats of a row of the sums
  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int c16 = lane & 15, q4 = lane >> 4;
  const int y = quot(block, a.by_Hkv), c = block - y * a.Hkv;
  const int unit = quot(y, a.few.by_splits), split = y - unit * a.few.splits;
  FewRows rows;
  if (!few_rows_of<BOTH>(a, unit, lane, rows)) return;
  const SeqRows sr = rows.sr;
  const int b = sr.b, n_rows = rows.i1, p_first = uni(sr.kv - sr.n);

  const uint64_t k_head = reinterpret_cast<uint64_t>(a.kc) + c * a.kc_h * kEsz;
  const uint64_t v_head = reinterpret_cast<uint64_t>(a.vc) + c * a.vc_h * kEsz;
  const uint64_t ke_head = reinterpret_cast<uint64_t>(a.ke) + c * a.ke_h, ve_head = reinterpret_cast<uint64_t>(a.ve) + c * a.ve_h;
  const uint32_t k_lane = (uint32_t)(c16 * (int)a.kc_t * kEsz + 16 * q4), v_lane = (uint32_t)(c16 * (int)a.vc_t * kEsz + 16 * q4);
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

  for (int i0 = rows.i0; i0 < n_rows; i0 += 16 * NQ) {
    const int p_lo = uni(p_first + quot(i0, a.by_r)), p_hi = uni(p_first + quot(min(i0 + 16 * NQ, n_rows) - 1, a.by_r));
    const KeyTiles kt = key_tiles<TK>(a.window, a.sinks, p_lo, p_hi, sr.keys);
    const Piece piece = pieces_of(a.few, kt.total);
    const int per = piece.per, n0 = split * per, n1 = uni(min(kt.total, n0 + per));
    if (split > 0 && n0 >= n1) continue;

    struct Ahead {   // what is known of a tile before its loads go out
      CacheRow row[2];
      Groups<2> groups;
    };
    auto rows_of = [&](int n, CacheRow (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int j = kt.tile(n) * TK + 16 * kb + c16;
        x[kb] = cache_row(a, b, j, n < n1 && is_seen(a, p_lo, kt.end, j));
      }
    };
    auto look_up = [&](int n, Ahead& x) __attribute__((always_inline)) {
      if constexpr (BY16) x.groups = groups_of<2>(a, b, kt.tile(max(min(n, n1 - 1), 0)) * TK);
      else rows_of(n, x.row);
    };
    auto load = [&](T& t, const Ahead& x, int n) __attribute__((always_inline)) {
      const uint64_t zero = zero_address();
      int j0 = 0;
      if constexpr (BY16) {
        j0 = kt.tile(max(min(n, n1 - 1), 0)) * TK;
        t.seen = n < n1 ? seen_of<2>(a, x.groups, p_lo, kt.end, j0) : 0;
      } else {
        t.seen = ((uint32_t)__builtin_amdgcn_ballot_w64(x.row[0].page >= 0) & 0xffffu) |
                 ((uint32_t)__builtin_amdgcn_ballot_w64(x.row[1].page >= 0) << 16);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        uint64_t kp, vp, ke = zero, ve = zero;
        if constexpr (BY16) {
          const int page = x.groups.page[kb], at = place_of(a, j0 + 16 * kb);
          const bool there = t.seen >> (16 * kb + c16) & 1;
          kp = there ? k_head + (page * a.kc_p + at * a.kc_t) * kEsz + k_lane : zero + 16 * q4;
          vp = there ? v_head + (page * a.vc_p + at * a.vc_t) * kEsz + v_lane : zero + 16 * q4;
          if constexpr (E4M3) {
            ke = there ? ke_head + page * a.ke_p + at * a.ke_t + (uint32_t)(c16 * (int)a.ke_t) : zero;
            ve = there ? ve_head + page * a.ve_p + at * a.ve_t + (uint32_t)(c16 * (int)a.ve_t) : zero;
          }
        } else {
          const CacheRow r = x.row[kb];
          const bool there = r.page >= 0;
          kp = (there ? k_head + (r.page * a.kc_p + r.at * a.kc_t) * kEsz : zero) + 16 * q4;
          vp = (there ? v_head + (r.page * a.vc_p + r.at * a.vc_t) * kEsz : zero) + 16 * q4;
          if constexpr (E4M3) {
            ke = there ? ke_head + r.page * a.ke_p + r.at * a.ke_t : zero;
            ve = there ? ve_head + r.page * a.ve_p + r.at * a.ve_t : zero;
          }
        }
#pragma unroll
        for (int i = 0; i < T::N; ++i) t.k[kb][i] = load16(kp + 64 * i);
#pragma unroll
        for (int i = 0; i < T::N; ++i) t.v[kb][i] = load16(vp + 64 * i);
        if constexpr (E4M3) {
          t.ks[kb] = load_scale(ke);
          t.vs[kb] = load_scale(ve);
        }
      }
    };

    // this wave's tiles: n0 + w, n0 + w + 4, ..
    // The look-up of a tile goes out ahead of the loads of the tile before it, so that waiting for it is not waiting for them.
    T ta, tb;
    Ahead at{}, at_next{};
    look_up(n0 + w, at);
    look_up(n0 + w + kWaves, at_next);
    load(ta, at, n0 + w);

    bf16x8 qf[NQ][KF];
    int pos[NQ], n_seen[NQ];
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      const int row = min(i0 + 16 * qb + c16, n_rows - 1), tq = quot(row, a.by_r), h = c * a.r + row - tq * a.r;
      pos[qb] = min(p_first + tq, sr.keys - 1);
      n_seen[qb] = keys_up_to(a.window, p_first + tq, pos[qb]);
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
      at = at_next;
      look_up(n + 2 * kWaves, at_next);
      if constexpr (NQ == 1) load(nxt, at, n + kWaves);   // (past the end: zeros)
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
            *reinterpret_cast<u32x4*>(Vs + Tile<D>::off(16 * kb + c16, q4 + 4 * i)) = cur.v[kb][i];
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
      if constexpr (NQ > 1) load(nxt, at, n + kWaves);
      const bool masked = j0 + TK - 1 > p_lo || ~seen != 0 || (a.window > 0 && j0 < p_hi - a.window + 1);
      const uint32_t seen_l = seen >> (4 * q4);
      const int sinks = a.window > 0 ? a.sinks : 0;
      bf16x8 pf[NQ];
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[kb][qb][e] *= c2;
        if (masked) {
          int d0 = pos[qb] - j0 - 4 * q4;
          asm volatile("" : "+v"(d0));
          const int last = min(pos[qb], sinks - 1) - j0 - 4 * q4;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int bit = 16 * kb + e;
              const bool in = (((unsigned)(d0 - bit) < (unsigned)n_seen[qb]) | (bit <= last)) & (seen_l >> bit & 1);
              sc[kb][qb][e] = in ? sc[kb][qb][e] : -INFINITY;
            }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, sc[kb][qb][e]);
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
    const PArgs z = BOTH ? late_args() : a;
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
      const int tq = quot(i0 + row, z.by_r), h = c * z.r + i0 + row - tq * z.r, t = sr.s0 + tq, H = z.Hkv * z.r;
      if (piece.count > 1) {
        const size_t dst = part_row(z, z.few, z.few_slots, split, b, c, i0 + row, t, h);
        f32x4* po = reinterpret_cast<f32x4*>(z.few.part_o + dst * D + 8 * ch);
        po[0] = s0 * inv;
        po[1] = s1 * inv;
        if (ch == 0) z.few.part_lse[dst] = lse2;
      } else {
        *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(z.o) + ((size_t)t * H + h) * D + 8 * ch) = pack8(s0 * inv, s1 * inv);
        if (ch == 0 && z.lse) z.lse[(size_t)h * z.T + t] = lse2 * kLn2;
      }
    }
    if constexpr (NQ > 1) return;   // 32 rows at most: no other turn
    __syncthreads();                // before the next rows' V
  }
}

template <int D>
constexpr int kChunkBytes = 4 * kKeys * Tile<D>::kRow;
template <int D, int NQ>
constexpr int kFewBytes = 4 * 16 * NQ * (D + 4 + 2) * 4 > 4 * 32 * D * 2 ? 4 * 16 * NQ * (D + 4 + 2) * 4 : 4 * 32 * D * 2;

template <int D, bool E4M3, bool BY16>
__global__ void __launch_bounds__(256, 2) paged_chunk_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kChunkBytes<D>];
  __shared__ int flags[4];
  chunk_workgroup<D, E4M3, BY16>(a, first_block + block_id(), smem, flags);
}

template <int D, bool E4M3, bool BY16, int NQ>
__global__ void __launch_bounds__(256, 2) paged_few_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kFewBytes<D, NQ>];
  few_workgroup<D, E4M3, BY16, NQ, false>(a, first_block + block_id(), smem);
}

template <int D, bool E4M3, bool BY16>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) paged_both_kernel(PArgs a, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[kChunkBytes<D> > kFewBytes<D, 1> ? kChunkBytes<D> : kFewBytes<D, 1>];
  __shared__ int flags[4];
  const int block = first_block + block_id();
  if (block < a.chunk_blocks)   // the long chains first: 62 us, the others first 72 (16 sequences of 1 to 600 rows, window 4096)
    chunk_workgroup<D, E4M3, BY16>(a, block, smem, flags);
  else
    few_workgroup<D, E4M3, BY16, 1, true>(a, block - a.chunk_blocks, smem);
}

template <int D, bool E4M3, bool BY16>
int launch_t(const PArgs& a, int nq, hipStream_t st) {
  const int few = a.few.n_tiles * a.Hkv * a.few.splits;
  if (a.chunk_blocks == 0) {
    if constexpr (E4M3)
      if (nq == 2) return launch_blocks(paged_few_kernel<D, E4M3, BY16, 2>, few, 256, st, a);
    return launch_blocks(paged_few_kernel<D, E4M3, BY16, 1>, few, 256, st, a);
  }
  if constexpr (D == 128 && BY16) {
    if (a.chunk_rows == 256) {
      const int rc = launch_blocks(paged_long_kernel<E4M3>, a.chunk_blocks, 512, st, a);
      return rc != 0 || a.few_rows == 0 ? rc : launch_blocks(paged_few_kernel<D, E4M3, BY16, 1>, few, 256, st, a);
    }
  }
  if (a.few_rows == 0) return launch_blocks(paged_chunk_kernel<D, E4M3, BY16>, a.chunk_blocks, 256, st, a);
  return launch_blocks(paged_both_kernel<D, E4M3, BY16>, a.chunk_blocks + few, 256, st, a);
}
template <int D, bool E4M3>
int launch_pages(const PArgs& a, int nq, hipStream_t st) {
  return a.by16 ? launch_t<D, E4M3, true>(a, nq, st) : launch_t<D, E4M3, false>(a, nq, st);
}

}  // namespace

int launch_paged_bf16(const PArgs& a, int D, bool e4m3, int nq, hipStream_t st) {
  if (D == 64) return e4m3 ? launch_pages<64, true>(a, nq, st) : launch_pages<64, false>(a, nq, st);
  return e4m3 ? launch_pages<128, true>(a, nq, st) : launch_pages<128, false>(a, nq, st);
}

}  // namespace s2
