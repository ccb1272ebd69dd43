// bf16 S2-Attn forward for gfx950: tiled online-softmax attention inside each group
// of LongLoRA Section 3.2, with the shift of Algorithm 1 folded into row addresses.
//
// One workgroup (4 waves) owns 128 consecutive query rows of one (batch, head, group)
// in the head's rolled frame; a wave owns 32 of them.  It walks the 64-key tiles of
// the same group up to the diagonal.  Per tile and wave:
//   S^T = K Q^T        A = K rows from LDS (row-major fragments), B = Q^T in registers
//   online softmax     queries are lane-indexed, keys register-indexed, so row max and
//                      row sum are in-lane reductions plus one exchange with lane^32;
//                      the running maximum is only raised (and O rescaled) when it
//                      grows by more than 2^8, which keeps exp2 arguments <= 8
//   O^T += V^T P^T     A = V^T through transposing LDS reads, B = P^T straight from the
//                      S^T accumulators (no cross-lane movement)
// K/V tiles go global -> LDS directly (global_load_lds, 16 bytes per lane) into two
// stages, one barrier per tile.  The output tile is transposed through LDS and stored
// with 16-byte coalesced writes at the un-rolled token rows.
#include "s2attn_bf16_common.h"
#include "s2attn_bf16_fwd.h"
#include "s2attn_device.h"
#include "s2attn_launch.h"

namespace s2 {
namespace {

// Removes what query row `qrow` does not see under a window: key <= qrow and qrow - key < window in one comparison.  One way
// through and not two (tiles without sinks by themselves): the compiler then moves the scores to other registers.
__device__ __forceinline__ void mask_window(f32x16& s0, f32x16& s1, int j0, int qrow, const Win& win, int g32) {
  int d0 = qrow - j0 - 4 * g32;
  asm volatile("" : "+v"(d0));   // keeps the compiler from doing all this ahead of the branch that asks for it
  const unsigned n = win.window;
  const int last = min(qrow, win.sinks - 1) - j0 - 4 * g32;   // keys up to it are sinks that the row sees
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int bit = 8 * (v >> 2) + (v & 3);
    s0[v] = (((unsigned)(d0 - bit) < n) | (bit <= last)) ? s0[v] : -INFINITY;
    s1[v] = (((unsigned)(d0 - bit - 32) < n) | (bit + 32 <= last)) ? s1[v] : -INFINITY;
  }
}

// Normalises a wave's 32 x 128 output block, transposes it through the wave's private
// 8 KB LDS region and stores it (and lse) at the un-rolled token rows.
template <bool RAGGED>
__device__ __forceinline__ void fwd_epilogue(const KArgs& a, FwdState& st, char* Os, int b, int h, const Run& run, int s,
                                             int qw0, float c2, int lane, int l32, int g32) {
  const float l_tot = sum_halves(st.l_run);
  const float inv = 1.f / l_tot;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int vv = 0; vv < 4; ++vv) {
      const bf16x4 pk = pack4(st.o_acc[db][4 * vv] * inv, st.o_acc[db][4 * vv + 1] * inv,
                              st.o_acc[db][4 * vv + 2] * inv, st.o_acc[db][4 * vv + 3] * inv);
      *reinterpret_cast<bf16x4*>(Os + tile_off(l32, 4 * db + vv) + 8 * g32) = pk;
    }
  wave_lds_order();
  store_wave_rows<RAGGED>(a, a.o, a.so, Os, run, qw0, s, b, h, lane);
  if (g32 == 0 && (!RAGGED || qw0 + l32 < run.len)) {
    const int tok = token_of(run.p0 + qw0 + l32, s, a.N);
    a.lse[((size_t)b * a.H + h) * a.N + tok] = (st.m_run * c2 + __builtin_amdgcn_logf(l_tot)) * kLn2;
  }
}

// RAGGED: G is not a multiple of 128, the shift not of 64 or a Variant 2 split not of 128 --
// tiles may be partial and the wrap point may fall inside one; the rows of such a tile find
// their tokens one by one, all other tiles are 64 consecutive tokens.  The two halves of a
// split wrap-around group run as causal runs of their own (run_of_tile).
// WINDOW (with RAGGED): one run of all tokens, key tiles of the sinks and of the window.
template <bool RAGGED, bool WINDOW>
__device__ __forceinline__ void fwd_workgroup(const KArgs& a, int T, const Deal& deal, int block, const Win& win, char* smem) {
  constexpr int BM = 128;
  const int tid = thread_id(), lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;

  // ---- block -> (batch, head, group, query tile): every XCD walks its own sequences, the query
  // heads of a kv head back to back and the tiles of a sequence heaviest first, so that the K/V
  // of a group stay in that XCD's L2 while they are being re-read.  The sequences are dealt out
  // per query head and not per kv head: with one kv head and four groups the latter gave work to
  // four of the eight XCDs only (N = 8192, H = 32, G = 2048: forward 278 us,
  // 149 dealt out per query head; dQ 383 and 198).
  int seq, rank, qt;
  if constexpr (WINDOW) {
    if (!decode_stretch<true>(win, win.cut_q, win.by_cut_q, block, T, deal, seq, qt)) return;
  } else {
    if (!decode_block(block, T, deal, seq, rank)) return;
    qt = T - 1 - rank;
  }
  const HeadPos at = head_of_seq(a, seq);
  const int gidx = at.g, c = at.c, b = at.b, h = at.h;

  const int s = uni(shift_of_head(a, h));
  // the causal run this block works in and the first row of the other block of a split
  // wrap-around group inside it (aligned kernels skip whole tiles at `split`; the ragged
  // ones run the two blocks as runs of their own and see no split)
  Run run{gidx * a.G, a.G};
  int split = uni(split_of_group(a, gidx, s));
  if constexpr (RAGGED) {
    if (!run_of_tile(a, gidx, s, BM, qt, run)) return;
    run.p0 = uni(run.p0); run.len = uni(run.len);
    split = run.len;
  }
  const int i0 = qt * BM;
  const int qw0 = i0 + w * 32;                      // first query row of this wave
  const int qrow = qw0 + l32;
  const int lo_w = uni(qw0 >= split ? split : 0);        // first key visible to this wave
  const int jt_first = uni((i0 >= split ? split : 0) / BN);
  const int jt_diag = i0 / BN;                      // tiles jt_diag, jt_diag + 1 touch the diagonal
  const float c2 = a.scale_log2;

  const __bf16* qp = static_cast<const __bf16*>(a.q);
  const char* kp = static_cast<const char*>(a.k);
  const char* vp = static_cast<const char*>(a.v);

  // ---- Q^T fragments of this wave, straight from global memory
  bf16x8 qf[8];
  {
    const int tok = run_token(a, run, qrow, s);
    const bf16x8* src = reinterpret_cast<const bf16x8*>(qp + row_off(a.sq, b, tok, h));
#pragma unroll
    for (int st = 0; st < 8; ++st) qf[st] = src[2 * st + g32];
  }

  // ---- K/V staging, global -> LDS: wave w, pass p fills tile rows 16p + 4w .. +3
  // (1 KB contiguous in LDS); lane i lands on physical chunk i%16 of row i/16 and
  // therefore fetches the logical chunk that the swizzle places there.
  const int st_row = 4 * w + (lane >> 4);
  const uint64_t k_row_bytes = (uint64_t)a.sk.t * 2, v_row_bytes = (uint64_t)a.sv.t * 2;
  const uint32_t smem_base = lds_addr(smem);
  const uint32_t st_chunk = (uint32_t)(((lane & 15) ^ swz(st_row)) << 4);
  // aligned staging: scalar base of the tile's 64-token run plus these per-lane offsets
  const uint32_t k_lane = (uint32_t)(st_row * k_row_bytes) + st_chunk;
  const uint32_t v_lane = (uint32_t)(st_row * v_row_bytes) + st_chunk;
  const uint64_t k_head = uni64(reinterpret_cast<uint64_t>(kp) + row_off(a.sk, b, 0, c) * 2);
  const uint64_t v_head = uni64(reinterpret_cast<uint64_t>(vp) + row_off(a.sv, b, 0, c) * 2);
  auto issue_tile = [&](int jt, int stage) {
    const uint32_t ks = smem_base + stage * 2 * kTileBytes + 4 * w * kRowBytes;
    const int row0 = jt * BN;
    const uint32_t tok0 = (uint32_t)token_of(run.p0 + row0, s, a.N);
    if (RAGGED && (row0 + BN > run.len || (int)tok0 + BN > a.N)) {
      // not 64 consecutive tokens: row by row, rows past the end of the run repeat its last row
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int tok = run_token(a, run, row0 + 16 * p + st_row, s);
        dma16(kp + row_off(a.sk, b, tok, c) * 2 + st_chunk, ks + 16 * p * kRowBytes);
        dma16(vp + row_off(a.sv, b, tok, c) * 2 + st_chunk, ks + 16 * p * kRowBytes + kTileBytes);
      }
      return;
    }
    const uint64_t kb = k_head + tok0 * k_row_bytes, vb = v_head + tok0 * v_row_bytes;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      dma16s(kb + p * 16 * k_row_bytes, k_lane, ks + 16 * p * kRowBytes);
      dma16s(vb + p * 16 * v_row_bytes, v_lane, ks + 16 * p * kRowBytes + kTileBytes);
    }
  };

  LaneOffsets lo;
  init_lane_offsets(lo, lane);
  FwdState st;
  st.m_run = -INFINITY;
  st.l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) st.o_acc[db] = zero16();

  if constexpr (WINDOW) {
    st.m_run = first_max(c2);   // a row may see nothing of the first tiles
    const KeyTiles kt = key_tiles<BN>(win.window, win.sinks, i0, i0 + BM - 1, a.N);
    issue_tile(kt.tile(0), 0);
    for (int n = 0; n < kt.total; ++n) {
      const int stage = n & 1, j0 = kt.tile(n) * BN;
      wait_vmcnt0();
      __syncthreads();
      if (n + 1 < kt.total) issue_tile(kt.tile(n + 1), stage ^ 1);
      const char* Ks = smem + stage * 2 * kTileBytes;
      // after the wave's rows, or between the sinks and their windows
      if (j0 > qw0 + 31 || qw0 >= a.N || (j0 + BN <= qw0 - win.window + 1 && j0 >= win.sinks)) continue;
      f32x16 s0, s1;
      bf16x8 pf[4];
      fwd_scores(s0, s1, qf, Ks, lo, j0, qrow, g32, false);
      if (j0 + BN - 1 > qw0 || j0 < qw0 + 31 - win.window + 1) mask_window(s0, s1, j0, qrow, win, g32);
      fwd_softmax(st, s0, s1, c2, pf);
      fwd_pv(st, Ks + kTileBytes, lo, pf);
    }
    __syncthreads();
    fwd_epilogue<RAGGED>(a, st, smem + w * (32 * kRowBytes), b, h, run, s, qw0, c2, lane, l32, g32);
    return;
  }

  issue_tile(jt_first, 0);
  const int n_tiles = jt_diag + 2 - jt_first;
  for (int n = 0; n < n_tiles; ++n) {
    const int jt = jt_first + n;
    const int stage = n & 1;
    wait_vmcnt0();                        // this wave's part of tile jt has landed
    __syncthreads();                      // everyone's part has landed; everyone left tile jt-1
    if (n + 1 < n_tiles) issue_tile(jt + 1, stage ^ 1);
    const int j0 = jt * BN;
    const char* Ks = smem + stage * 2 * kTileBytes;
    const char* Vs = Ks + kTileBytes;
    // this wave's rows see keys [lo_w, row]: skip tiles wholly outside (beyond the
    // diagonal, or, under Variant 2, in the other block of the wrap group)
    if (j0 > qw0 + 31 || j0 + BN - 1 < lo_w) continue;
    fwd_tile(st, qf, Ks, Vs, lo, j0, qrow, c2, g32, j0 + BN - 1 > qw0);
  }
  __syncthreads();

  // ---- epilogue: normalise, transpose through LDS, store at un-rolled token rows
  fwd_epilogue<RAGGED>(a, st, smem + w * (32 * kRowBytes), b, h, run, s, qw0, c2, lane, l32, g32);
}

template <bool RAGGED>
__global__ void __launch_bounds__(256, 2)
fwd_bf16_kernel(KArgs a, int T, Deal deal, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[4 * kTileBytes];   // [stage][K,V]
  fetch_args(a, deal);
  fwd_workgroup<RAGGED, false>(a, T, deal, first_block + block_id(), Win{}, smem);
}

__global__ void __launch_bounds__(256, 2)
window_fwd_bf16_kernel(KArgs a, int T, Deal deal, Win win, int first_block) {
  __shared__ __attribute__((aligned(1024))) char smem[4 * kTileBytes];
  fwd_workgroup<true, true>(a, T, deal, first_block + block_id(), win, smem);
}

__device__ __forceinline__ void mask_scores(f32x16& s0, f32x16& s1, int j0, int qrow, int g32) {
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int key = j0 + 8 * (v >> 2) + 4 * g32 + (v & 3);
    if (key > qrow) s0[v] = -INFINITY;
    if (key + 32 > qrow) s1[v] = -INFINITY;
  }
}

// ---------------------------------------------------------------------------
// Eight-wave variant (groups of 2048 and more): a workgroup owns 256 query rows and keeps
// three K/V stages in LDS, one workgroup per CU, two waves per SIMD.  Each wave runs
// the tile loop software-pipelined across tiles: the matrix block of an iteration is
// P(n) V(n) followed by S(n+1) = K(n+1) Q^T, the vector block is the softmax of one
// tile.  Waves 0-3 run the vector block after the matrix block, waves 4-7 before it,
// so the two waves that share a SIMD alternate between the matrix and vector units
// instead of competing for them ("ping-pong"), with a single barrier per tile.
// RAGGED: tiles of 256 rows that are not full, a wrap point inside a tile or a split off the tiles;
// only the key tiles that are not 64 consecutive tokens are staged row by row.
// ---------------------------------------------------------------------------
template <bool RAGGED>
__global__ void __launch_bounds__(512, 1)
fwd_bf16_pp_kernel(KArgs a, int T, Deal deal) {
  constexpr int BM = 256;
  constexpr int kStageBytes = 2 * kTileBytes;
  __shared__ __attribute__((aligned(1024))) char smem[3 * kStageBytes];   // [stage][K,V]
  fetch_args(a, deal);

  const int tid = thread_id(), lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  const int grp = w >> 2;

  int seq, rank;
  if (!decode_block(block_id(), T, deal, seq, rank)) return;
  const HeadPos at = head_of_seq(a, seq);
  const int gidx = at.g, c = at.c, b = at.b, h = at.h;
  int qt = T - 1 - rank;

  const int s = uni(shift_of_head(a, h));
  Run run{gidx * a.G, a.G};
  int split = uni(split_of_group(a, gidx, s));
  if constexpr (RAGGED) {
    if (!run_of_tile(a, gidx, s, BM, qt, run)) return;
    qt = uni(qt); run.p0 = uni(run.p0); run.len = uni(run.len);
    split = run.len + BM;   // no split inside a run
  }
  const int i0 = qt * BM;
  const int qw0 = i0 + w * 32;
  const int qrow = qw0 + l32;
  const int jt_first = uni((i0 >= split ? split : 0) / BN);     // first tile any wave needs
  const int nt = uni((RAGGED ? min(i0 + BM, run.len) - 1 : i0 + BM - 1) / BN - jt_first + 1);   // tiles the workgroup walks
  // this wave's own tile range, relative to jt_first
  const int n_lo = uni((qw0 >= split ? split : 0) / BN - jt_first);
  const int n_hi = uni(RAGGED && qw0 >= run.len ? -1 : (qw0 + 31) / BN - jt_first);   // -1: padding rows only
  const float c2 = a.scale_log2;

  const __bf16* qp = static_cast<const __bf16*>(a.q);
  const char* kp = static_cast<const char*>(a.k);
  const char* vp = static_cast<const char*>(a.v);

  bf16x8 qf[8];
  {
    const int tok = run_token(a, run, qrow, s);
    const bf16x8* src = reinterpret_cast<const bf16x8*>(qp + row_off(a.sq, b, tok, h));
#pragma unroll
    for (int st = 0; st < 8; ++st) qf[st] = src[2 * st + g32];
  }

  // staging: wave w, pass p fills tile rows 32p + 4w .. +3 of K and of V.  A tile is a
  // contiguous run of 64 tokens, so its address is a scalar (head base + first token) plus a
  // per-lane offset (row within the pass, swizzled chunk) that never changes.
  const int st_row = 4 * w + (lane >> 4);
  const uint64_t k_row_bytes = (uint64_t)a.sk.t * 2, v_row_bytes = (uint64_t)a.sv.t * 2;
  const uint32_t smem_base = lds_addr(smem);
  const uint32_t st_chunk = (uint32_t)(((lane & 15) ^ swz(st_row)) << 4);
  const uint32_t k_lane = (uint32_t)(st_row * k_row_bytes) + st_chunk;
  const uint32_t v_lane = (uint32_t)(st_row * v_row_bytes) + st_chunk;
  const uint64_t k_head = uni64(reinterpret_cast<uint64_t>(kp) + row_off(a.sk, b, 0, c) * 2);
  const uint64_t v_head = uni64(reinterpret_cast<uint64_t>(vp) + row_off(a.sv, b, 0, c) * 2);
  auto issue_tile = [&](int n, int stage) {
    const int row0 = (jt_first + n) * BN;
    const uint32_t tok0 = (uint32_t)token_of(run.p0 + row0, s, a.N);
    const uint32_t ks = smem_base + stage * kStageBytes + 4 * w * kRowBytes;
    if (RAGGED && (row0 + BN > run.len || (int)tok0 + BN > a.N)) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int tok = run_token(a, run, row0 + 32 * p + st_row, s);
        dma16(kp + row_off(a.sk, b, tok, c) * 2 + st_chunk, ks + 32 * p * kRowBytes);
        dma16(vp + row_off(a.sv, b, tok, c) * 2 + st_chunk, ks + 32 * p * kRowBytes + kTileBytes);
      }
      return;
    }
    const uint64_t kb = k_head + tok0 * k_row_bytes, vb = v_head + tok0 * v_row_bytes;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      dma16s(kb + p * 32 * k_row_bytes, k_lane, ks + 32 * p * kRowBytes);
      dma16s(vb + p * 32 * v_row_bytes, v_lane, ks + 32 * p * kRowBytes + kTileBytes);
    }
  };

  LaneOffsets lo;
  init_lane_offsets(lo, lane);
  FwdState st;
  st.m_run = first_max(c2);
  st.l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) st.o_acc[db] = zero16();
  f32x16 s0, s1;       // scores of the tile whose softmax is pending
  bf16x8 pf[4];        // probabilities of the tile whose PV product is pending
  bf16x8 ring[4][4];   // operand fragments of steps k, k+1, k+2 (slot = step mod 4)

  // ---- prologue: tiles 0 and 1 in flight, scores of tile 0
  issue_tile(0, 0);
  if (nt > 1) {
    issue_tile(1, 1);
    __builtin_amdgcn_s_waitcnt(0x0F74);   // vmcnt(4): tile 0 has landed, tile 1 may be in flight
  } else {
    wait_vmcnt0();
  }
  __syncthreads();
  if (n_lo <= 0 && 0 <= n_hi) {
    fwd_scores(s0, s1, qf, smem, lo, jt_first * BN, qrow, g32, jt_first * BN + BN - 1 > qw0);
    if (grp == 0) fwd_softmax(st, s0, s1, c2, pf);
    pp_load<0>(ring[0], smem + kTileBytes, nullptr, lo);     // first two steps of P(0) V(0)
    pp_load<1>(ring[1], smem + kTileBytes, nullptr, lo);
  }

  int st_cur = 0, st_nxt = 1, st_free = 2;   // stages of tile n, tile n+1, and the free one
  for (int n = 0; n < nt; ++n) {
    wait_vmcnt0();        // this wave's part of tile n+1 has landed
    __syncthreads();      // all of tile n+1 has landed; every wave has left tile n-1
    if (n + 2 < nt) issue_tile(n + 2, st_free);
    const bool act = n_lo <= n && n <= n_hi;
    const bool act_next = n + 1 < nt && n_lo <= n + 1 && n + 1 <= n_hi;
    const char* Vs_cur = smem + st_cur * kStageBytes + kTileBytes;
    const char* Ks_nxt = smem + st_nxt * kStageBytes;
    const char* Vs_nxt = Ks_nxt + kTileBytes;
    if (grp == 1 && act) fwd_softmax(st, s0, s1, c2, pf);
    // Every step issues the LDS reads of the step two ahead, then its own four MFMAs.  The
    // matrix block runs at raised priority so that it is not starved by the vector work of
    // the wave it shares the SIMD with.
    __builtin_amdgcn_s_setprio(1);
    if (act) {
      pp_load<2>(ring[2], Vs_cur, Ks_nxt, lo);
      pp_mma<0>(ring[0], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      pp_load<3>(ring[3], Vs_cur, Ks_nxt, lo);
      pp_mma<1>(ring[1], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      if (act_next) pp_load<4>(ring[0], Vs_cur, Ks_nxt, lo);
      pp_mma<2>(ring[2], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      if (act_next) pp_load<5>(ring[1], Vs_cur, Ks_nxt, lo);
      pp_mma<3>(ring[3], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (act_next) {
      if (!act) {   // this wave's first tile: nothing was prefetched
        pp_load<4>(ring[0], Vs_cur, Ks_nxt, lo);
        pp_load<5>(ring[1], Vs_cur, Ks_nxt, lo);
      }
      s0 = zero16();
      s1 = zero16();
      pp_load<6>(ring[2], Vs_cur, Ks_nxt, lo);
      pp_mma<4>(ring[0], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      pp_load<7>(ring[3], Vs_cur, Ks_nxt, lo);
      pp_mma<5>(ring[1], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      pp_load<0>(ring[0], Vs_nxt, nullptr, lo);     // first two steps of the next iteration
      pp_mma<6>(ring[2], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      pp_load<1>(ring[1], Vs_nxt, nullptr, lo);
      pp_mma<7>(ring[3], st, pf, qf, s0, s1);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      const int j0 = (jt_first + n + 1) * BN;
      if (j0 + BN - 1 > qw0) mask_scores(s0, s1, j0, qrow, g32);
      if (grp == 0) fwd_softmax(st, s0, s1, c2, pf);
    }
    __builtin_amdgcn_s_setprio(0);
    const int t = st_cur; st_cur = st_nxt; st_nxt = st_free; st_free = t;
  }
  __syncthreads();
  fwd_epilogue<RAGGED>(a, st, smem + w * (32 * kRowBytes), b, h, run, s, qw0, c2, lane, l32, g32);
}

// Eight waves under a window: one run of all tokens, the key tiles of the sinks and of the window.
__global__ void __launch_bounds__(512, 1)
window_fwd_bf16_pp_kernel(KArgs a, int T, Deal deal, Win win) {
  constexpr int BM = 256;
  __shared__ __attribute__((aligned(1024))) char smem[3 * 2 * kTileBytes];   // [stage][K,V]
  const int tid = thread_id(), lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  int seq, qt;
  if (!decode_stretch<true>(win, win.cut_q, win.by_cut_q, block_id(), T, deal, seq, qt)) return;
  const HeadPos at = head_of_seq(a, seq);
  const int c = at.c, b = at.b, h = at.h;
  const int i0 = uni(qt * BM);
  const Run run{0, a.N};
  const int qw0 = i0 + w * 32, qrow = qw0 + l32;
  const KeyTiles kt = key_tiles<BN>(win.window, win.sinks, i0, i0 + BM - 1, a.N);
  const float c2 = a.scale_log2;

  bf16x8 qf[8];
  {
    const bf16x8* src = reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + row_off(a.sq, b, min(qrow, a.N - 1), h));
#pragma unroll
    for (int st = 0; st < 8; ++st) qf[st] = src[2 * st + g32];
  }
  const int st_row = 4 * w + (lane >> 4);
  const uint64_t k_row_bytes = (uint64_t)a.sk.t * 2, v_row_bytes = (uint64_t)a.sv.t * 2;
  const uint32_t smem_base = lds_addr(smem);
  const uint32_t st_chunk = (uint32_t)(((lane & 15) ^ swz(st_row)) << 4);
  const uint32_t k_lane = (uint32_t)(st_row * k_row_bytes) + st_chunk;
  const uint32_t v_lane = (uint32_t)(st_row * v_row_bytes) + st_chunk;
  const uint64_t k_head = uni64(reinterpret_cast<uint64_t>(a.k) + row_off(a.sk, b, 0, c) * 2);
  const uint64_t v_head = uni64(reinterpret_cast<uint64_t>(a.v) + row_off(a.sv, b, 0, c) * 2);
  auto issue = [&](int n, int stage) __attribute__((always_inline)) {
    const uint32_t row0 = kt.tile(n) * BN;
    const uint32_t ks = smem_base + stage * 2 * kTileBytes + 4 * w * kRowBytes;
    if ((int)row0 + BN > a.N) {   // rows past the end repeat the last row
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint64_t tok = min((int)row0 + 32 * p + st_row, a.N - 1);
        dma16(reinterpret_cast<const char*>(k_head + tok * k_row_bytes + st_chunk), ks + 32 * p * kRowBytes);
        dma16(reinterpret_cast<const char*>(v_head + tok * v_row_bytes + st_chunk), ks + 32 * p * kRowBytes + kTileBytes);
      }
      return;
    }
    const uint64_t kb = k_head + row0 * k_row_bytes, vb = v_head + row0 * v_row_bytes;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      dma16s(kb + p * 32 * k_row_bytes, k_lane, ks + 32 * p * kRowBytes);
      dma16s(vb + p * 32 * v_row_bytes, v_lane, ks + 32 * p * kRowBytes + kTileBytes);
    }
  };
  LaneOffsets lo;
  init_lane_offsets(lo, lane);
  FwdState st;
  st.m_run = first_max(c2);
  st.l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) st.o_acc[db] = zero16();
  pp_walk(st, qf, lo, smem, kt.total, w >> 2, c2, issue, [](int) {},
          [&](int n) {   // not after the wave's rows, and not between the sinks and their windows
            const int j0 = kt.tile(n) * BN;
            return j0 <= qw0 + 31 && qw0 < a.N && (j0 + BN > qw0 - win.window + 1 || j0 < win.sinks);
          },
          [&](f32x16& s0, f32x16& s1, int n) {
            const int j0 = kt.tile(n) * BN;
            if (j0 + BN - 1 > qw0 || j0 < qw0 + 31 - win.window + 1) mask_window(s0, s1, j0, qrow, win, g32);
          });
  __syncthreads();
  fwd_epilogue<true>(a, st, smem + w * (32 * kRowBytes), b, h, run, 0, qw0, c2, lane, l32, g32);
}

}  // namespace

int launch_window_fwd_bf16(const KArgs& a, Win win, hipStream_t st) {
  if (a.D == 64) return launch_window_fwd_d64(a, win, st);
  // Eight waves only for long walks: of the tiles that 256 rows meet a wave's 32 need all but three or four, and one workgroup a
  // CU has nothing beside its first and last tile.  us, four waves and eight, N = 32768, H = 32, four sinks: window 1024 756
  // and 786, 2048 1252 and 1260, 4096 2193 and 2089, 8192 3833 and 3564; N = 4096 2048 131 and 127, 4096 146 and 137.
  if (win.window >= 4096) {
    const WindowGrid g = window_grid_q(win, ragged_tiles(a, 256), a.B * a.H, a.r, 32);
    hipLaunchKernelGGL(window_fwd_bf16_pp_kernel, dim3(g.grid.blocks), dim3(512), 0, st, a, g.T, g.grid.deal, win);
    return hipGetLastError() == hipSuccess ? 0 : -1;
  }
  const WindowGrid g = window_grid_q(win, ragged_tiles(a, 128), a.B * a.H, a.r, 64);
  return launch_blocks(window_fwd_bf16_kernel, g.grid.blocks, 256, st, a, g.T, g.grid.deal, win);
}

int launch_fwd_bf16(const KArgs& a, hipStream_t st) {
  if (a.D == 64) return launch_fwd_d64(a, st);
  if (fwd_is_small(a)) return launch_fwd_small(a, st);
  const int n_seq = a.B * a.H * a.NG;
  // groups of 2048 tokens or more: the eight-wave kernel; shorter tile sequences run a little
  // faster (4-9 % at G = 512 ... 1024) with two independent four-wave workgroups per CU, whose
  // prologues and epilogues overlap
  const bool partial = a.ragged || a.G % 256 != 0;   // tiles of 256 rows that are not full
  const int T8 = partial ? ragged_tiles(a, 256) : a.G / 256;
  // Tiles that are not full go there only with more than three workgroups to two CUs: up to then four
  // waves fill the chip better (G = 2050: 72 workgroups of eight waves 48.7 us, with four 42.0; 288 53.3 and
  // 51.1; 432 78.4 and 77.1; G = 4000: 256 91.8 and 88.3, 512 131 and 143).  And where 128 rows would divide the group
  // (G % 256 == 128), only from 4096 tokens on: the four-wave kernel then has no partial tile to test for
  // (H = 32, eight groups: G = 2688 553 and 512 us, 3200 740 and 715; G = 4224 602 and 603, 6016 1152 and
  // 1160, four groups of 10880 1774 and 1855).
  if (a.G >= 2048 && (!partial || (n_seq * (long long)T8 > 384 && (a.ragged || a.G >= 4096)))) {
    const Grid g = grid_of(T8, n_seq, a.r, 32);   // 32 CUs per XCD, one workgroup each
    if (partial)
      hipLaunchKernelGGL(fwd_bf16_pp_kernel<true>, dim3(g.blocks), dim3(512), 0, st, a, T8, g.deal);
    else
      hipLaunchKernelGGL(fwd_bf16_pp_kernel<false>, dim3(g.blocks), dim3(512), 0, st, a, T8, g.deal);
    return hipGetLastError() == hipSuccess ? 0 : -1;
  }
  const int T = a.ragged ? ragged_tiles(a, 128) : a.G / 128;
  const Grid g = grid_of(T, n_seq, a.r, 64, true);   // 32 CUs per XCD, two workgroups each
  if (a.ragged) return launch_blocks(fwd_bf16_kernel<true>, g.blocks, 256, st, a, T, g.deal);
  return launch_blocks(fwd_bf16_kernel<false>, g.blocks, 256, st, a, T, g.deal);
}

}  // namespace s2
