// Per-wave tile code of the bf16 forward kernels for head dimension 128: a wave's 32 queries against a 64-key tile in LDS
// (s2attn_bf16_fwd.hip says how the kernels use it).
#pragma once
#include "s2attn_bf16_common.h"

namespace s2 {
namespace {

constexpr int BN = 64;                       // keys per tile
constexpr int kTileBytes = BN * kRowBytes;   // 16 KB
constexpr float kRescaleThreshold = 8.f;     // log2 units

struct FwdState {
  f32x16 o_acc[4];
  float m_run;    // running row maximum (raw score units), shared by lanes l and l^32
  float l_run;    // this lane's part of the running row sum
};

// O^T += V^T P^T for the 16 keys starting at tile row KROW0.
template <int KROW0>
__device__ __forceinline__ void pv_step(FwdState& st, const char* Vs, const LaneOffsets& lo, bf16x8 pf) {
  bf16x8 vf[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) vf[db] = frag_tr<KROW0>(Vs, lo, db);
#pragma unroll
  for (int db = 0; db < 4; ++db) st.o_acc[db] = mfma32(vf[db], pf, st.o_acc[db]);
}

// S^T = K Q^T of one 64-key tile for one wave (32 queries): two 32-key blocks.
// `masked` is wave-uniform: the tile touches the diagonal of this wave's rows.
__device__ __forceinline__ void fwd_scores(f32x16& s0, f32x16& s1, const bf16x8 (&qf)[8], const char* Ks,
                                           const LaneOffsets& lo, int j0, int qrow, int g32, bool masked) {
  s0 = zero16();
  s1 = zero16();
  bf16x8 ka[4], kb[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ka[i] = frag_rm<0>(Ks, lo, i);
    kb[i] = frag_rm<32>(Ks, lo, i);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s0 = mfma32(ka[i], qf[i], s0);
    s1 = mfma32(kb[i], qf[i], s1);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ka[i] = frag_rm<0>(Ks, lo, i + 4);
    kb[i] = frag_rm<32>(Ks, lo, i + 4);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s0 = mfma32(ka[i], qf[i + 4], s0);
    s1 = mfma32(kb[i], qf[i + 4], s1);
  }
  if (masked) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = j0 + 8 * (v >> 2) + 4 * g32 + (v & 3);
      if (key > qrow) s0[v] = -INFINITY;
      if (key + 32 > qrow) s1[v] = -INFINITY;
    }
  }
}

// Online softmax of the tile: updates the running maximum lazily, accumulates the row
// sum and packs the probabilities as the four 16-key B operands of the PV product.
// The maximum of every tile is formed, sixteen instructions and a chain of ten.  Without it (a score far above the
// running maximum shows in the row sum, and only then is the maximum formed and the exponentials taken again) N(0, 1)
// inputs take 0.98 to 1.00 of the time, but others more, or P is rounded where it is not now: a row's largest P is 1 and
// exact if the maximum was raised for it.  With the line at a sum of 2^8, as here, scores of standard deviation 3
// take 1.04 of the time, of 8 1.12 (N = 8192, H = 32, G = 2048); at 2^12 of 8 1.05, and O is 5 % further from 64 bits at 16; at
// 2^32 none takes longer, and dq leaves its bound.
__device__ __forceinline__ void fwd_softmax(FwdState& st, f32x16& s0, f32x16& s1, float c2, bf16x8 (&pf)[4]) {
  // two independent three-input maximum chains
  float ma = fmaxf(s0[0], s0[1]), mb = fmaxf(s1[0], s1[1]);
#pragma unroll
  for (int v = 2; v < 16; v += 2) {
    ma = fmaxf(fmaxf(ma, s0[v]), s0[v + 1]);
    mb = fmaxf(fmaxf(mb, s1[v]), s1[v + 1]);
  }
  const float mx = max_halves(fmaxf(ma, mb));
  if (__builtin_amdgcn_ballot_w64(mx * c2 > st.m_run * c2 + kRescaleThreshold) != 0) {
    const float m_new = fmaxf(st.m_run, mx);
    const float alpha = __builtin_amdgcn_exp2f((st.m_run - m_new) * c2);
    st.m_run = m_new;
    st.l_run *= alpha;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) st.o_acc[db][v] *= alpha;
  }
  const float mc = st.m_run * c2;
  float ra = 0.f, rb = 0.f;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    s0[v] = __builtin_amdgcn_exp2f(fmaf(s0[v], c2, -mc));
    s1[v] = __builtin_amdgcn_exp2f(fmaf(s1[v], c2, -mc));
    ra += s0[v];
    rb += s1[v];
  }
  st.l_run += ra + rb;
  pf[0] = pack8(s0[0], s0[1], s0[2], s0[3], s0[4], s0[5], s0[6], s0[7]);
  pf[1] = pack8(s0[8], s0[9], s0[10], s0[11], s0[12], s0[13], s0[14], s0[15]);
  pf[2] = pack8(s1[0], s1[1], s1[2], s1[3], s1[4], s1[5], s1[6], s1[7]);
  pf[3] = pack8(s1[8], s1[9], s1[10], s1[11], s1[12], s1[13], s1[14], s1[15]);
}

// O^T += V^T P^T for the whole 64-key tile.
__device__ __forceinline__ void fwd_pv(FwdState& st, const char* Vs, const LaneOffsets& lo, const bf16x8 (&pf)[4]) {
  pv_step<0>(st, Vs, lo, pf[0]);
  pv_step<16>(st, Vs, lo, pf[1]);
  pv_step<32>(st, Vs, lo, pf[2]);
  pv_step<48>(st, Vs, lo, pf[3]);
}

__device__ __forceinline__ void fwd_tile(FwdState& st, const bf16x8 (&qf)[8], const char* Ks, const char* Vs,
                                         const LaneOffsets& lo, int j0, int qrow, float c2, int g32, bool masked) {
  f32x16 s0, s1;
  bf16x8 pf[4];
  fwd_scores(s0, s1, qf, Ks, lo, j0, qrow, g32, masked);
  fwd_softmax(st, s0, s1, c2, pf);
  fwd_pv(st, Vs, lo, pf);
}

// ---- the matrix block of the eight-wave kernel as 8 steps of 4 MFMAs, each fed by 4
// operand fragments.  Steps 0-3: O^T += V^T P^T for keys 16k .. 16k+15 of the current
// tile; steps 4-7: S^T += K Q^T over d = 32(k-4) .. +31 of the next tile.
template <int STEP>
__device__ __forceinline__ void pp_load(bf16x8 (&buf)[4], const char* Vs_cur, const char* Ks_nxt, const LaneOffsets& lo) {
  if constexpr (STEP < 4) {
#pragma unroll
    for (int db = 0; db < 4; ++db) buf[db] = frag_tr<16 * STEP>(Vs_cur, lo, db);
  } else {
    constexpr int J = STEP - 4;
    buf[0] = frag_rm<0>(Ks_nxt, lo, 2 * J);
    buf[1] = frag_rm<32>(Ks_nxt, lo, 2 * J);
    buf[2] = frag_rm<0>(Ks_nxt, lo, 2 * J + 1);
    buf[3] = frag_rm<32>(Ks_nxt, lo, 2 * J + 1);
  }
}

template <int STEP>
__device__ __forceinline__ void pp_mma(const bf16x8 (&buf)[4], FwdState& st, const bf16x8 (&pf)[4],
                                       const bf16x8 (&qf)[8], f32x16& s0, f32x16& s1) {
  if constexpr (STEP < 4) {
#pragma unroll
    for (int db = 0; db < 4; ++db) st.o_acc[db] = mfma32(buf[db], pf[STEP], st.o_acc[db]);
  } else {
    constexpr int J = STEP - 4;
    s0 = mfma32(buf[0], qf[2 * J], s0);
    s1 = mfma32(buf[1], qf[2 * J], s1);
    s0 = mfma32(buf[2], qf[2 * J + 1], s0);
    s1 = mfma32(buf[3], qf[2 * J + 1], s1);
  }
}

// The tile walk of the eight-wave kernels whose tiles and masks are not those of a causal run: the loop of fwd_bf16_pp_kernel
// over nt tiles.  issue(n, stage) starts the staging of tile n and land(n) ends that of tile n where it has to be ended by hand
// (LDS then holds it after the next barrier); act(n): the wave has work in tile n; mask(s0, s1, n) removes scores.
// smem: three stages of [K, V].
template <class Issue, class Land, class Act, class Mask>
__device__ __forceinline__ void pp_walk(FwdState& st, const bf16x8 (&qf)[8], const LaneOffsets& lo, char* smem, int nt, int grp, float c2,
                                        Issue issue, Land land, Act act_of, Mask mask) {
  constexpr int kStageBytes = 2 * kTileBytes;
  f32x16 s0, s1;       // scores of the tile whose softmax is pending
  bf16x8 pf[4];        // probabilities of the tile whose PV product is pending
  bf16x8 ring[4][4];   // operand fragments of steps k, k+1, k+2 (slot = step mod 4)
  if (nt <= 0) return;
  issue(0, 0);
  land(0);
  if (nt > 1) issue(1, 1);
  wait_vmcnt0();
  __syncthreads();
  bool act = act_of(0);
  if (act) {
    fwd_scores(s0, s1, qf, smem, lo, 0, 0, 0, false);
    mask(s0, s1, 0);
    if (grp == 0) fwd_softmax(st, s0, s1, c2, pf);
    pp_load<0>(ring[0], smem + kTileBytes, nullptr, lo);
    pp_load<1>(ring[1], smem + kTileBytes, nullptr, lo);
  }
  int st_cur = 0, st_nxt = 1, st_free = 2;   // stages of tile n, tile n+1, and the free one
  for (int n = 0; n < nt; ++n) {
    if (n + 1 < nt) land(n + 1);
    wait_vmcnt0();        // this wave's part of tile n+1 has landed
    __syncthreads();      // all of tile n+1 has landed; every wave has left tile n-1
    if (n + 2 < nt) issue(n + 2, st_free);
    const bool act_next = n + 1 < nt && act_of(n + 1);
    const char* Vs_cur = smem + st_cur * kStageBytes + kTileBytes;
    const char* Ks_nxt = smem + st_nxt * kStageBytes;
    const char* Vs_nxt = Ks_nxt + kTileBytes;
    if (grp == 1 && act) fwd_softmax(st, s0, s1, c2, pf);
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
      if (!act) {   // nothing was prefetched
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
      mask(s0, s1, n + 1);
      if (grp == 0) fwd_softmax(st, s0, s1, c2, pf);
    }
    __builtin_amdgcn_s_setprio(0);
    act = act_next;
    const int t = st_cur; st_cur = st_nxt; st_nxt = st_free; st_free = t;
  }
}

}  // namespace
}  // namespace s2
