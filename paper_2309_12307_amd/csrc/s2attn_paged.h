// What the kernels of the paged cache share: the argument block, how a block finds its sequence and how a key
// position finds its row in the cache.
//
// Nothing that these kernels read from the device is trusted with an address: row_start is clamped to [0, T], key positions
// stay below table_cols * page_size, and a page number outside [0, pages) stands for no page (its keys are invisible).
#pragma once
#include <type_traits>

#include "s2attn_device.h"

namespace s2 {

// How the work of a launch, or of a part of it, is dealt out.
struct PSet {
  int splits, min_tiles;                       // most pieces the keys of a row tile are cut into; fewest key tiles of one
  int n_tiles;                                 // row tiles (chunk), units (few)
  Div by_tiles, by_groups, by_splits, by_min;  // n_tiles, Hkv * splits, splits, min_tiles
  float* part_o; float* part_lse;              // splits > 1: [split][part_rows][D] and [split][part_rows] (base 2)
  long long part_rows;
};

struct PArgs {
  const void* q; void* o; float* lse;          // (T,H,D), (T,H,D), (H,T) or null
  void* k; void* v;                            // rows of the call, (T,Hkv,D): written to the cache or read from it
  char* kc; char* vc;                          // cache, (pages, page_size, Hkv, D)
  uint8_t* ke; uint8_t* ve;                    // e4m3: biased exponents, (pages, page_size, Hkv)
  const int* table; const int* row_start; const int* kv_len;
  long long q_t, q_h, k_t, k_h, v_t, v_h;      // strides in elements
  long long kc_p, kc_t, kc_h, vc_p, vc_t, vc_h;
  long long ke_p, ke_t, ke_h, ve_p, ve_t, ve_h;
  long long table_b;
  int T, B, H, Hkv, r, pages, page_size, max_keys;   // max_keys: table_cols * page_size
  int window, sinks;                           // window 0: every earlier key is visible
  PSet chunk, few;                             // sequences of more than few_rows (row, head of the kv head) pairs, and the others
  int few_rows, chunk_rows;                    // chunk_rows: of a row tile of `chunk`
  int few_slots;                               // rows of the pieces of `few`: few_rows of a sequence and kv head, not (T, H) (part_row)
  int few_tokens;                              // `few` deals out so many tokens of a sequence at a time (2^30: all of them)
  int by16;                                    // pages of a multiple of 16 tokens, 16 rows of one within 31-bit offsets
  int chunk_blocks;                            // blocks of `chunk`; those of `few` follow
  Div by_r, by_page, by_Hkv, by_few_tokens;
  float scale_log2;
};

// The arguments again, as the kernels' first, for what is used only once a workgroup's keys are done: read from memory then, and not kept
// in scalar registers (or spilled from them) until then.
__device__ __forceinline__ PArgs late_args() {
  auto p = (const __attribute__((address_space(4))) void*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  PArgs a;
  __builtin_memcpy(&a, (const void*)p, sizeof(a));
  return a;
}

__device__ __forceinline__ int wave_uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int start_of(const PArgs& a, int i) { return min(max(a.row_start[i], 0), a.T); }

// Rows of sequence b: packed rows s0 .. s0 + n - 1, the positions kv - n .. kv - 1; keys: cached positions that exist.
struct SeqRows {
  int b, s0, n, kv, keys;
};
__device__ __forceinline__ SeqRows seq_rows(const PArgs& a, int b) {
  SeqRows s;
  s.b = b;
  s.s0 = start_of(a, b);
  s.n = max(start_of(a, b + 1) - s.s0, 0);
  s.kv = max(a.kv_len[b], 0);
  s.keys = min(s.kv, a.max_keys);
  return s;
}

// The last sequence whose first unit is at or before `id` (b = -1: none): units are packed rows (SHIFT < 0) or row
// tiles of 2^SHIFT (token, query head of the kv head) pairs, of which a sequence owns those from
// (row_start[b] * r >> SHIFT) + b on: at least as many as it needs, and no running sum is needed to place them.
// The whole wave calls it and has one answer: up to 64 sequences are looked at together, everything about them read at once;
// more are narrowed down by looking at every 64th part first.  Where row_start falls, the answer is some sequence.
template <int SHIFT>
__device__ __forceinline__ int first_tile(const PArgs& a, int s0, int b) { return (int)((unsigned)(s0 * a.r) >> SHIFT) + b; }
template <int SHIFT>
__device__ __forceinline__ SeqRows find_rows(const PArgs& a, int id, int lane) {
  auto before = [&](int start, int i) __attribute__((always_inline)) {
    const int s0 = min(max(start, 0), a.T);
    if constexpr (SHIFT < 0) return s0 <= id;
    else return first_tile<SHIFT>(a, s0, i) <= id;
  };
  int lo = 0, hi = a.B;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) >> 6, i = lo + lane * step;
    const int m = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < hi && before(a.row_start[min(i, hi - 1)], i)));
    lo += max(wave_uniform(m) - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  const int i = min(lo + lane, hi - 1);
  const int start = a.row_start[i], end = a.row_start[i + 1], kv = a.kv_len[i];
  const int l = wave_uniform(__builtin_popcountll(__builtin_amdgcn_ballot_w64(lo + lane < hi && before(start, i)))) - 1;
  SeqRows s;
  s.b = l < 0 ? -1 : lo + l;
  s.s0 = min(max(__builtin_amdgcn_readlane(start, max(l, 0)), 0), a.T);
  s.n = max(min(max(__builtin_amdgcn_readlane(end, max(l, 0)), 0), a.T) - s.s0, 0);
  s.kv = max(__builtin_amdgcn_readlane(kv, max(l, 0)), 0);
  s.keys = min(s.kv, a.max_keys);
  return s;
}

// Rows i0 .. i1 - 1 of a sequence's (token, query head of the kv head) pairs: those of a workgroup of `few`, by turns where it holds fewer.
struct FewRows {
  SeqRows sr;
  int i0, i1;
};
// The rows of unit u < B: those of the first few_tokens tokens of sequence u, if they are few_rows or less.  Its other tokens, which a
// step of single tokens does not have, are units behind those: unit B + j - 1 has the few_tokens ones that begin in the j-th few_tokens
// rows of the call (one stretch of a sequence but its first does, at most).
template <bool BOTH>   // beside `chunk`: u < B, and all tokens
__device__ __forceinline__ bool few_rows_of(const PArgs& a, int u, int lane, FewRows& x) {
  if (u >= a.few.n_tiles) return false;
  int tok = 0;
  if (BOTH || u < a.B) {
    x.sr = seq_rows(a, u);
  } else {
    const int t0 = (u - a.B + 1) * a.few_tokens, t1 = min(t0 + a.few_tokens, a.T) - 1;
    for (int t = t0;; t = t1) {   // the sequences of the first and of the last of them
      x.sr = find_rows<-1>(a, t, lane);
      tok = x.sr.b < 0 ? 0 : quot(max(min(t1 - x.sr.s0, x.sr.n - 1), 0), a.by_few_tokens) * a.few_tokens;
      if (tok > 0 && x.sr.s0 + tok >= t0) break;
      if (t == t1) return false;
    }
  }
  x.i0 = wave_uniform(tok * a.r);
  x.i1 = wave_uniform((BOTH ? x.sr.n : min(tok + a.few_tokens, x.sr.n)) * a.r);
  return x.i1 <= a.few_rows;
}

// Row of a piece for query head h of token t, the i-th of its sequence's and kv head's rows.
__device__ __forceinline__ size_t part_row(const PArgs& a, const PSet& set, bool slots, int split, int b, int c, int i, int t, int h) {
  return (size_t)split * set.part_rows + (slots ? ((size_t)b * a.few_rows + i) * a.Hkv + c : (size_t)t * (a.Hkv * a.r) + h);
}

// Block -> (row tile, kv head, split).  Blocks of one (kv head, split) read the same keys: whole such groups go to an XCD
// where they divide among the eight, row tiles from the last (most keys) to the first.
__device__ __forceinline__ bool tile_of_block(const PArgs& a, const PSet& set, int block, int& tile, int& c, int& split) {
  const int groups = a.Hkv * set.splits;
  int g;
  if ((groups & 7) == 0) {
    const int slot = block >> 3, u = quot(slot, set.by_tiles);
    g = u * 8 + (block & 7);
    tile = slot - u * set.n_tiles;
  } else {
    tile = quot(block, set.by_groups);
    g = block - tile * groups;
  }
  tile = set.n_tiles - 1 - tile;
  split = quot(g, a.by_Hkv);
  c = g - split * a.Hkv;
  return tile >= 0 && g < groups;
}

// Pieces that the `total` key tiles of a row tile are cut into (at most `splits`, of min_tiles tiles or more in the mean), and
// the tiles of one: even ones.
struct Piece {
  int count, per;
};
__device__ __forceinline__ Piece pieces_of(const PSet& set, int total) {
  Piece x{1, total};
  if (set.splits > 1) {
    x.count = max(min(set.splits, quot(total, set.by_min)), 1);
    x.per = (total + x.count - 1) / x.count;
    x.count = x.per > 0 ? (total + x.per - 1) / x.per : 1;
  }
  return x;
}

// Of the keys before `end`, the rows of a tile from position p_lo on see all but those between the sinks and their windows: pages
// there may have been given up, and their memory may be anything.
__device__ __forceinline__ bool is_seen(const PArgs& a, int p_lo, int end, int j) {
  const int lo = a.window > 0 ? p_lo - a.window + 1 : 0;
  return (j < end) & ((j >= lo) | (j < a.sinks));
}

// The cache row of key position j, if it is wanted: page number (-1: none) and place in the page.
struct CacheRow {
  int page, at;
};
__device__ __forceinline__ CacheRow cache_row(const PArgs& a, int b, int j, bool wanted) {
  CacheRow x{-1, 0};
  if (wanted) {
    const int slot = quot(j, a.by_page);
    x.at = j - slot * a.page_size;
    const int page = a.table[b * a.table_b + slot];
    x.page = (unsigned)page < (unsigned)a.pages ? page : -1;
  }
  return x;
}

// Keys that a row sees up to `pos` without the sinks: all, or those of its window (pos is less than its position p_row where the
// sequence is cut off).
__device__ __forceinline__ int keys_up_to(int window, int p_row, int pos) {
  return max(window > 0 ? pos - max(p_row - window, -1) : pos + 1, 0);
}

// Where pages are of a multiple of 16 tokens, 16 keys from a multiple of 16 on lie in one page, one after the other: one look-up
// on the scalar unit and no address arithmetic a lane.  Page numbers of the N such groups of a tile.
template <int N>
struct Groups {
  int page[N];
};
template <int N>
__device__ __forceinline__ Groups<N> groups_of(const PArgs& a, int b, int j0) {
  Groups<N> x;
#pragma unroll
  for (int g = 0; g < N; ++g) x.page[g] = a.table[b * a.table_b + quot(min(j0 + 16 * g, a.max_keys - 1), a.by_page)];
  return x;
}
// The place in its page of key j0.
__device__ __forceinline__ int place_of(const PArgs& a, int j0) { return j0 - quot(j0, a.by_page) * a.page_size; }
// Bytes from a cache's first row (of a head) to place `at` of page `page`, all factors below 2^32 where a.by16.
__device__ __forceinline__ uint64_t group_off(int page, int at, long long page_bytes, long long token_bytes) {
  return (uint64_t)(uint32_t)page * (uint32_t)page_bytes + (uint32_t)at * (uint32_t)token_bytes;
}
// A bit a key for 16 N keys, and the first n of them.
template <int N>
using KeyBits = std::conditional_t<N == 2, uint32_t, uint64_t>;
template <int N>
__device__ __forceinline__ KeyBits<N> bits_below(int n) { return n >= 16 * N ? ~KeyBits<N>{0} : n <= 0 ? 0 : (KeyBits<N>{1} << n) - 1; }
// A bit for each of the 16 N keys from j0 on that exists and that some row of the tile sees (is_seen).
template <int N>
__device__ __forceinline__ KeyBits<N> seen_of(const PArgs& a, const Groups<N>& x, int p_lo, int end, int j0) {
  KeyBits<N> seen = 0;
#pragma unroll
  for (int g = 0; g < N; ++g)
    if ((unsigned)x.page[g] < (unsigned)a.pages) seen |= KeyBits<N>{0xffff} << (16 * g);
  const int lo = a.window > 0 ? p_lo - a.window + 1 : 0;
  if (j0 < lo || j0 + 16 * N > end) seen &= bits_below<N>(end - j0) & (~bits_below<N>(lo - j0) | bits_below<N>(a.sinks - j0));
  return seen;
}

// Tiles [from, n1) of TK keys of a walk lie on pages that exist and before `end`: their loads need no test.  The tiles of the sinks and
// the first of the window stay out: not all of their keys are seen.  The whole workgroup of THREADS looks.
struct Plain {
  int from, to;
};
template <int TK, int THREADS>
__device__ __forceinline__ Plain plain_tiles(const PArgs& a, int b, const KeyTiles& kt, int n0, int n1, int tid, int* flags) {
  Plain x;
  x.from = a.window > 0 ? max(n0, kt.n_sink + 1) : n0;
  x.to = min(n1, kt.n_sink + kt.end / TK - kt.first);   // (the last tile may reach past `end`)
  bool bad = false;
  if (x.from < x.to) {
    const int first = quot(kt.tile(x.from) * TK, a.by_page), last = quot(kt.tile(x.to - 1) * TK + TK - 1, a.by_page);
    const int* row = a.table + b * a.table_b;
    for (int s = first + tid; s <= last; s += 4 * THREADS)
#pragma unroll
      for (int u = 0; u < 4; ++u) bad |= (unsigned)row[min(s + u * THREADS, last)] >= (unsigned)a.pages;
  }
  const bool wave_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
  if ((tid & 63) == 0) flags[tid >> 6] = wave_bad;
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) any |= flags[w];
  if (wave_uniform(any)) x.to = x.from;
  return x;
}

// What stands for a row that is not there.
static __device__ const uint4 zero_row[32] = {};

// Loads from addresses that are global memory, said so: a choice between the cache and zero_row otherwise becomes a flat load,
// which waits for LDS too.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#define S2_GLOBAL(T, p) (*(const __attribute__((address_space(1))) T*)(p))
__device__ __forceinline__ uint64_t zero_address() { return reinterpret_cast<uint64_t>(&zero_row[0]); }
__device__ __forceinline__ u32x4 load16(uint64_t p) { return S2_GLOBAL(u32x4, p); }
__device__ __forceinline__ float load_scale(uint64_t p) { return __uint_as_float((uint32_t)S2_GLOBAL(uint8_t, p) << 23); }

}  // namespace s2
