// bf16 attention of new tokens over a paged cache (bf16 or e4m3) for gfx950.
//
// The rows of one sequence and kv head are its (token, query head of the kv head) pairs, token by token, so that K and V
// are read once for all query heads that share them.  A workgroup (4 waves) owns 128 of them and a piece of their keys; a
// wave owns 32.  It walks the 64-key tiles that any of its rows sees: S^T = K Q^T, online softmax, O^T += V^T P^T as
// in the forward kernels on contiguous tensors.  Rows that several pieces share leave normalised fp32 partial outputs and
// their log-sum-exp, which a second kernel joins.
//
// P is rounded to bf16 for the second product (as everywhere in this library); the row sum adds the unrounded P, and
// statistics, outputs and partial outputs stay fp32 up to the one rounding of o.
#include "s2attn_bf16_tile.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace s2 {
namespace {

constexpr int kKeys = 64;       // of a tile
constexpr int kRowsLog2 = 7;
constexpr int kRows = 1 << kRowsLog2;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Sixteen e4m3 values times 2^(exps - 127) as bf16: exact, the products have four significant bits.
__device__ __forceinline__ void widen(const uint4& u, float scale, bf16x8& lo, bf16x8& hi) {
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

template <int D, bool E4M3>
__global__ void __launch_bounds__(256, 2) paged_bf16_kernel(PArgs a, int first_block) {
  using L = Tile<D>;
  constexpr int kTileBytes = kKeys * L::kRow;
  constexpr int KS = D / 16, DB = D / 32, kChunks = D / 8;      // k-steps, column blocks, 16-byte chunks of a bf16 row
  constexpr int kEsz = E4M3 ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) char smem[4 * kTileBytes];   // [stage][K, V]

  const int tid = thread_id(), lane = tid & 63, w = uni(tid >> 6);
  const int g32 = lane >> 5, l32 = lane & 31;
  int tile, c, split;
  if (!tile_of_block(a, first_block + block_id(), tile, c, split)) return;
  const int b = find_seq<kRowsLog2>(a, tile, lane);
  if (b < 0) return;
  const SeqRows sr = seq_rows(a, b);
  const int i0 = uni((tile - first_tile<kRowsLog2>(a, b)) * kRows), n_rows = uni(sr.n * a.r);
  if (i0 >= n_rows) return;
  const int p_first = uni(sr.kv - sr.n);                        // position of the sequence's first row
  const int p_lo = uni(p_first + quot(i0, a.by_r));
  const int p_hi = uni(p_first + quot(min(i0 + kRows, n_rows) - 1, a.by_r));
  const KeyTiles kt = key_tiles<kKeys>(a.window, a.sinks, p_lo, p_hi, sr.keys);
  const int per = tiles_of_split(a, kt.total);
  const int n0 = split * per, n1 = uni(min(kt.total, n0 + per));
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

  CacheRow next = look_up(n0);
  uint64_t seen = 0, seen_next = 0;
  if (n0 < n1) {
    seen_next = seen_of(next);
    issue(next, 0);
    land(0);
    next = look_up(n0 + 1);
  }
  for (int n = n0; n < n1; ++n) {
    const int stage = (n - n0) & 1;
    wait_vmcnt0();                        // this wave's part of tile n has landed
    __syncthreads();                      // everyone's part has landed; everyone left tile n - 1
    seen = seen_next;
    if (n + 1 < n1) {
      seen_next = seen_of(next);
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
        const int first = windowed ? p_first + tq - a.window + 1 : 0;
        const uint32_t seen0 = (uint32_t)seen >> (4 * g32), seen1 = (uint32_t)(seen >> 32) >> (4 * g32);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int bit = 8 * (v >> 2) + (v & 3), key = j0 + 4 * g32 + bit;
          if (!(key <= pos && (key >= first || key < a.sinks) && (seen0 >> bit & 1))) s0[v] = -INFINITY;
          if (!(key + 32 <= pos && (key + 32 >= first || key + 32 < a.sinks) && (seen1 >> bit & 1))) s1[v] = -INFINITY;
        }
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
    if (n + 1 < n1) land(stage ^ 1);
  }
  __syncthreads();

  // ---- o / l and the log-sum-exp; a row that saw nothing: 0 and -inf
  const float l_tot = sum_halves(l_run);
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  const float lse2 = l_tot == 0.f ? -INFINITY : m_run * c2 + __builtin_amdgcn_logf(l_tot);
  if (idle) return;
  const bool valid = iw + l32 < n_rows;
  const int H = a.Hkv * a.r;
  if (kt.total > per) {   // a piece
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
  char* region = smem + w * 32 * L::kRow;
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
      *reinterpret_cast<uint4*>(static_cast<__bf16*>(a.o) + ((size_t)(sr.s0 + ti) * H + hi) * D + ch * 8) = val[it];
    }
  }
  if (g32 == 0 && valid && a.lse) a.lse[(size_t)h * a.T + t] = lse2 * kLn2;
}

template <int D>
int launch_t(const PArgs& a, int cache, int blocks, hipStream_t st) {
  if (cache == 2) return launch_blocks(paged_bf16_kernel<D, true>, blocks, 256, st, a);
  return launch_blocks(paged_bf16_kernel<D, false>, blocks, 256, st, a);
}

}  // namespace

int launch_paged_bf16(const PArgs& a, int D, int cache, int blocks, hipStream_t st) {
  return D == 64 ? launch_t<64>(a, cache, blocks, st) : launch_t<128>(a, cache, blocks, st);
}

}  // namespace s2
