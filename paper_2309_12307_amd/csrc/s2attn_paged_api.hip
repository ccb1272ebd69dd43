// Host side of the paged cache's entry points (include/s2attn.h): argument checks, how finely the keys are dealt out,
// and launches.  Nothing here allocates device memory.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "s2attn.h"
#include "s2attn_launch.h"
#include "s2attn_paged.h"

namespace {

constexpr size_t kAlign = 256;
constexpr long long kMost = 1LL << 30;   // key positions of a sequence, (row, head) pairs of a call

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

struct Axis {
  long long stride, extent;
};

// Strides of a tensor whose axes have these extents, the contiguous ones where all are zero; `last` elements are
// contiguous.
template <int N>
void resolve(const long long (&st)[N], const long long (&extent)[N], long long last, long long (&out)[N]) {
  bool zero = true;
  for (long long x : st) zero = zero && x == 0;
  long long step = last;
  for (int i = N - 1; i >= 0; --i) {
    out[i] = zero ? step : st[i];
    step *= extent[i];
  }
}

// No stride negative, off `align` or too long for 64-bit offsets; distinct rows in distinct places where `disjoint`.
template <int N>
bool strides_ok(const long long (&st)[N], const long long (&extent)[N], long long last, int align, bool disjoint) {
  long long s[N];
  resolve(st, extent, last, s);
  Axis ax[N];
  for (int i = 0; i < N; ++i) {
    if (s[i] < 0 || s[i] % align != 0 || s[i] >= (1LL << 40)) return false;
    if (extent[i] > 1 && (double)s[i] * extent[i] > 4.0e18) return false;
    ax[i] = Axis{s[i], extent[i]};
  }
  if (!disjoint) return true;
  std::sort(ax, ax + N, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
  long long span = last;
  for (const Axis& x : ax) {
    if (x.extent <= 1) continue;
    if (x.stride < span) return false;
    span = x.stride * (x.extent - 1) + span;
  }
  return true;
}

int bytes_of(int dtype) { return dtype == S2ATTN_F32 ? 4 : dtype == S2ATTN_BF16 ? 2 : 1; }

bool shape_valid(const s2attn_paged_params* p) {
  return p->T >= 0 && p->B > 0 && p->H > 0 && p->Hkv > 0 && p->D > 0 && p->pages > 0 && p->page_size > 0 && p->table_cols > 0;
}

int tile_keys(const s2attn_paged_params* p) { return p->dtype == S2ATTN_F32 ? 32 : 64; }

long long row_tiles(const s2attn_paged_params* p, int rows) { return (long long)p->T * (p->H / p->Hkv) / rows + p->B; }

// Which sequences go to which kind of workgroup, and into how many pieces their keys are cut at most.
struct Plan {
  bool chunk, few;
  int chunk_rows;              // of a row tile of `chunk`
  int nq, few_rows;            // 16-row blocks of a `few` workgroup; the most rows of a sequence that goes there
  int few_tokens;              // tokens of a sequence dealt out at a time there
  int chunk_splits, chunk_min; // pieces, key tiles of a piece at least
  int few_splits, few_min;
};
Plan plan(const s2attn_paged_params* p, bool by16) {
  Plan x{};
  const long long r = p->H / p->Hkv, rows = p->T * r, seqs = std::max(1, std::min(p->B, p->T));
  // One token a sequence (as far as T and B tell), of up to 16 rows (e4m3 32 in two blocks, fp32 64 in turns): all go to `few`, by as many
  // tokens as a turn takes: a sequence that has several after all, among empty slots, has workgroups for all of them (256 rows of one
  // of 256 sequences over 8192 keys, H = 64, Hkv = 8, D = 128: 0.60 ms; by turns of one workgroup to a kv head 16.0; as the only
  // sequence, in `chunk`, 0.09).  Rows that are few in all go there by turns.  Where some sequences have more, those of up to 16
  // rows (fp32 64) go there and the others to `chunk`.  us, all in `chunk` and all in `few`, 4000 keys, D = 128: fp32, one sequence of 16
  // rows 35.8 and 19.9, of 64 65.9 and 57.2, eight of 16 78 and 56; bf16, one of 16 15.2 and 14.6, of 24 15.6 and 15.9, eight of 20
  // 30.5 and 43.6; e4m3, one of 24 20.4 and 15.4, eight of 20 32 and 39; one token of 32 sequences, H = 32, bf16 290 and 272, 16 over
  // 30 000 keys, e4m3 558 and 300.
  const bool f32 = p->dtype == S2ATTN_F32, e4m3 = p->cache_dtype == S2ATTN_E4M3;
  const long long most_few = f32 ? 64 : e4m3 ? 32 : 16;
  x.nq = 1;
  x.few_tokens = (int)kMost;
  if ((p->T <= p->B && r <= most_few) || rows <= most_few) {
    x.few = true;
    if (!f32 && (p->T <= p->B ? r : rows) > 16) x.nq = 2;
    x.few_rows = INT_MAX;
    if (p->T <= p->B) x.few_tokens = std::max(1, 16 * x.nq / (int)r);
  } else {
    x.chunk = true;
    x.few_rows = f32 ? 64 : 16;
    x.few = p->B > 1 && r <= x.few_rows;   // (else one token is more)
    if (!x.few) x.few_rows = 0;
  }
  const long long most = (long long)p->table_cols * p->page_size;
  long long keys = p->max_kv > 0 ? std::min<long long>(p->max_kv, most) : most;
  if (p->window > 0) keys = std::min<long long>(keys, (long long)p->window + p->sinks + (rows + seqs - 1) / seqs + 128);
  auto pieces = [&](long long blocks, long long target, long long min_keys) {
    const long long n = std::min((keys + min_keys - 1) / min_keys, (target + blocks - 1) / blocks);
    return (int)std::max<long long>(1, std::min<long long>(n, 256));
  };
  // Eight waves on 256 rows where the sequences are long, if their tiles fill the chip or their pieces are long too.  us, four waves and
  // eight, H = 32: one sequence of 4096 rows over 8000 keys 417 and 410, of 2048 over 32 000 (Hkv = 8) 1002 and 933; of 1024 over 8000 (two
  // pieces) 151 and 146, of 512 (four) 90 and 93; H = 40, two of 700 over 3000 126 and 101; H = 8, eight of 512 over 4000 (two pieces) 90 and 116.
  const long long wide = (rows + 255) / 256 * p->Hkv;
  x.chunk_rows = f32 ? 64 : by16 && p->D == 128 && rows / seqs >= 512 && (wide >= 192 || keys * wide / 256 >= 4000) ? 256 : 128;
  const long long tile = x.chunk_rows, in_tile = std::min(tile, (rows + seqs - 1) / seqs);
  const long long tiles = std::max((rows + tile - 1) / tile, seqs);
  const long long min_keys = std::max<long long>(256, 8 * in_tile);
  // As many pieces as the chip holds workgroups of the longest sequences' keys; shorter ones get pieces of about that length, not as
  // many.  us, pieces of min_keys and of these: 16 sequences of 1 to 600 rows over up to 12 000 tokens, D = 64, in 512 workgroups
  // 321, in 768 257 and 226; one row over 30 000 tokens, 16 sequences, e4m3 304 and 299; over 4000, 128 sequences 168 and 163;
  // over 8192, 32 sequences 76.2 and 77.5.
  const int resident = in_tile <= 16 ? 2048 : x.chunk_rows == 256 ? 256 : p->D == 64 ? 768 : 512;
  x.chunk_splits = x.chunk ? pieces(tiles * p->Hkv, resident, min_keys) : 1;
  x.chunk_min = (int)(std::max(min_keys, keys / x.chunk_splits * 3 / 4) / tile_keys(p));
  x.few_splits = x.few ? pieces(seqs * p->Hkv, 2048, 256) : 1;
  x.few_min = (int)(std::max<long long>(256, keys / x.few_splits / 2) / (f32 ? 16 : 32));
  return x;
}

// Where the pieces' outputs go.  A piece of the rows of the call has room for all of them, (T, H) rows; sequences of few rows that are in
// more pieces than the others have slots of their own instead, few_rows a sequence and kv head, where that is less:
// the others may be prompts of any length.
struct Room {
  bool slots;
  size_t piece, slot_piece;    // bytes of a piece
  size_t wanted;
};
Room room(const s2attn_paged_params* p, const Plan& x) {
  Room y{};
  const size_t row = (p->D + 1) * sizeof(float);
  y.piece = (size_t)p->T * p->H * row;
  const int most = std::max(x.chunk_splits, x.few_splits);
  y.wanted = most > 1 ? most * y.piece : 0;
  if (x.chunk && x.few_splits > 1) {
    y.slot_piece = (size_t)p->B * x.few_rows * p->Hkv * row;
    size_t apart = x.few_splits * y.slot_piece;
    // beside pieces of all rows in whole ones, so that workspace_bytes / piece is the number that a workspace holds
    if (x.chunk_splits > 1) apart = (x.chunk_splits + (apart + y.piece - 1) / y.piece) * y.piece;
    y.slots = apart < y.wanted;
    if (y.slots) y.wanted = apart;
  }
  return y;
}

int check(const s2attn_paged_params* p, int call) {
  if (!p) return S2ATTN_ERR_NULL;
  if (call < S2ATTN_PAGED_WRITE || call > S2ATTN_PAGED_FWD) return S2ATTN_ERR_DTYPE;
  const bool fwd = call == S2ATTN_PAGED_FWD;
  if (p->dtype != S2ATTN_BF16 && p->dtype != S2ATTN_F32) return S2ATTN_ERR_DTYPE;
  if (p->cache_dtype != p->dtype && p->cache_dtype != S2ATTN_E4M3) return S2ATTN_ERR_DTYPE;
  const int H = fwd ? p->H : p->Hkv;
  if (p->T < 0 || p->B <= 0 || H <= 0 || p->Hkv <= 0 || p->D <= 0 || p->pages <= 0 || p->page_size <= 0 || p->table_cols <= 0)
    return S2ATTN_ERR_DIM;
  if (H % p->Hkv != 0) return S2ATTN_ERR_HEADS;
  if (p->D != 64 && p->D != 128) return S2ATTN_ERR_HEADDIM;
  if (fwd && (p->window < 0 || p->sinks < 0 || p->max_kv < 0)) return S2ATTN_ERR_WINDOW;
  // positions, (row, head) pairs and block numbers are non-negative ints; a wave's pieces of a row are counted in them too
  if ((long long)p->table_cols * p->page_size > kMost || (long long)p->T * H > kMost || p->Hkv > 65536) return S2ATTN_ERR_TOO_LARGE;
  if ((long long)p->T * p->Hkv > kMost / 8 || p->B > (1 << 24)) return S2ATTN_ERR_TOO_LARGE;
  if (fwd && row_tiles(p, 64) * p->Hkv > kMost / 2) return S2ATTN_ERR_TOO_LARGE;

  const int row_align = 16 / bytes_of(p->dtype), cache_align = 16 / bytes_of(p->cache_dtype);
  const long long cache_ext[3] = {p->pages, p->page_size, p->Hkv}, kv_ext[2] = {p->T, p->Hkv}, q_ext[2] = {p->T, H};
  const bool write = call == S2ATTN_PAGED_WRITE, read = call == S2ATTN_PAGED_READ, e4m3 = p->cache_dtype == S2ATTN_E4M3;
  if (!strides_ok(p->k_cache_strides, cache_ext, p->D, cache_align, write) || !strides_ok(p->v_cache_strides, cache_ext, p->D, cache_align, write))
    return S2ATTN_ERR_STRIDE;
  if (e4m3 && (!strides_ok(p->k_exp_strides, cache_ext, 1, 1, write) || !strides_ok(p->v_exp_strides, cache_ext, 1, 1, write)))
    return S2ATTN_ERR_STRIDE;
  if (p->table_stride != 0 && p->B > 1 && (p->table_stride < 0 || p->table_stride >= (1LL << 40))) return S2ATTN_ERR_STRIDE;
  if (fwd ? !strides_ok(p->q_strides, q_ext, p->D, row_align, false)
          : !strides_ok(p->k_strides, kv_ext, p->D, row_align, read) || !strides_ok(p->v_strides, kv_ext, p->D, row_align, read))
    return S2ATTN_ERR_STRIDE;
  for (const void* x : {(const void*)p->page_table, (const void*)p->row_start, (const void*)p->kv_len}) {
    if (!x) return S2ATTN_ERR_NULL;
    if (!aligned(x, 4)) return S2ATTN_ERR_ALIGN;
  }
  for (const void* x : {p->k_cache, p->v_cache}) {
    if (!x) return S2ATTN_ERR_NULL;
    if (!aligned(x, 16)) return S2ATTN_ERR_ALIGN;
  }
  if (e4m3 && (!p->k_exp || !p->v_exp)) return S2ATTN_ERR_NULL;
  if (p->T > 0)
    for (const void* x : {fwd ? p->q : p->k, (const void*)(fwd ? p->o : p->v)}) {
      if (!x) return S2ATTN_ERR_NULL;
      if (!aligned(x, 16)) return S2ATTN_ERR_ALIGN;
    }
  if (fwd && !aligned(p->lse, 4)) return S2ATTN_ERR_ALIGN;
  if (fwd && p->workspace && !aligned(p->workspace, kAlign)) return S2ATTN_ERR_ALIGN;
  return S2ATTN_OK;
}

// 16 keys of a group lie in one page, and offsets within a page, of pages and of the rows of a group fit the arithmetic on the
// scalar unit.
bool groups_of_16(const s2attn_paged_params* p, const s2::PArgs& a) {
  if (p->page_size % 16 != 0) return false;
  const long long esz = bytes_of(p->cache_dtype), page = std::max(a.kc_p, a.vc_p) * esz, token = std::max(a.kc_t, a.vc_t) * esz;
  const long long exps = p->cache_dtype == S2ATTN_E4M3 ? std::max(a.ke_t, a.ve_t) : 0;
  return std::max(token, exps) < (1LL << 31) / 16 && std::max(page, token * p->page_size) < (1LL << 32);
}

s2::PArgs make_args(const s2attn_paged_params* p, int H) {
  s2::PArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = p->q; a.o = p->o; a.lse = p->lse; a.k = p->k; a.v = p->v;
  a.kc = static_cast<char*>(p->k_cache); a.vc = static_cast<char*>(p->v_cache);
  a.ke = p->k_exp; a.ve = p->v_exp;
  a.table = p->page_table; a.row_start = p->row_start; a.kv_len = p->kv_len;
  const long long cache_ext[3] = {p->pages, p->page_size, p->Hkv}, kv_ext[2] = {p->T, p->Hkv}, q_ext[2] = {p->T, H};
  long long s2[2], s3[3];
  resolve(p->q_strides, q_ext, p->D, s2); a.q_t = s2[0]; a.q_h = s2[1];
  resolve(p->k_strides, kv_ext, p->D, s2); a.k_t = s2[0]; a.k_h = s2[1];
  resolve(p->v_strides, kv_ext, p->D, s2); a.v_t = s2[0]; a.v_h = s2[1];
  resolve(p->k_cache_strides, cache_ext, p->D, s3); a.kc_p = s3[0]; a.kc_t = s3[1]; a.kc_h = s3[2];
  resolve(p->v_cache_strides, cache_ext, p->D, s3); a.vc_p = s3[0]; a.vc_t = s3[1]; a.vc_h = s3[2];
  resolve(p->k_exp_strides, cache_ext, 1, s3); a.ke_p = s3[0]; a.ke_t = s3[1]; a.ke_h = s3[2];
  resolve(p->v_exp_strides, cache_ext, 1, s3); a.ve_p = s3[0]; a.ve_t = s3[1]; a.ve_h = s3[2];
  a.table_b = p->table_stride != 0 ? p->table_stride : p->table_cols;
  a.T = p->T; a.B = p->B; a.Hkv = p->Hkv; a.r = H / p->Hkv;
  a.pages = p->pages; a.page_size = p->page_size; a.max_keys = p->table_cols * p->page_size;
  a.window = p->window >= kMost ? 0 : p->window;   // no position is that far from another
  a.sinks = p->sinks;
  a.by_Hkv = s2::div_by(p->Hkv);
  a.by16 = groups_of_16(p, a);
  a.by_r = s2::div_by(a.r);
  a.by_page = s2::div_by(a.page_size);
  a.scale_log2 = (p->scale > 0.f ? p->scale : 1.0f / std::sqrt((float)p->D)) * 1.4426950408889634f;
  return a;
}

int launched(int rc) { return rc == 0 ? S2ATTN_OK : S2ATTN_ERR_LAUNCH; }

}  // namespace

extern "C" {

int s2attn_check_paged_args(const s2attn_paged_params* p, int call) { return check(p, call); }

size_t s2attn_paged_workspace_bytes(const s2attn_paged_params* p) {
  if (!p || !shape_valid(p) || p->H % p->Hkv != 0) return 0;
  return room(p, plan(p, make_args(p, p->H).by16)).wanted;
}

int s2attn_cache_write(const s2attn_paged_params* p, void* stream) {
  int rc = check(p, S2ATTN_PAGED_WRITE);
  if (rc == S2ATTN_OK) rc = s2::check_device();
  if (rc != S2ATTN_OK || p->T == 0) return rc;
  return launched(s2::launch_cache_write(make_args(p, p->Hkv), p->D, p->dtype, p->cache_dtype, static_cast<hipStream_t>(stream)));
}

int s2attn_cache_read(const s2attn_paged_params* p, void* stream) {
  int rc = check(p, S2ATTN_PAGED_READ);
  if (rc == S2ATTN_OK) rc = s2::check_device();
  if (rc != S2ATTN_OK || p->T == 0) return rc;
  return launched(s2::launch_cache_read(make_args(p, p->Hkv), p->D, p->dtype, p->cache_dtype, static_cast<hipStream_t>(stream)));
}

int s2attn_paged_fwd(const s2attn_paged_params* p, void* stream) {
  int rc = check(p, S2ATTN_PAGED_FWD);
  if (rc == S2ATTN_OK) rc = s2::check_device();
  if (rc != S2ATTN_OK || p->T == 0) return rc;
  s2::PArgs a = make_args(p, p->H);
  const Plan x = plan(p, a.by16);
  // the pieces that the workspace holds: in one area, or slots, which get what the others leave but half of it at least, and the others
  const Room y = room(p, x);
  const size_t bytes = p->workspace ? p->workspace_bytes : 0;
  char* ws = static_cast<char*>(p->workspace);
  size_t few_bytes = 0;
  long long fit_chunk = bytes / y.piece, fit_few = fit_chunk;
  if (y.slots) {
    const size_t others = x.chunk_splits > 1 ? x.chunk_splits * y.piece : 0;
    fit_few = std::min<long long>(x.few_splits, std::max(bytes / 2, bytes - std::min(bytes, others)) / y.slot_piece);
    if (fit_few > 1) few_bytes = fit_few * y.slot_piece;
    fit_chunk = (bytes - few_bytes) / y.piece;
  }
  auto set = [&](s2::PSet& s, int n_tiles, int splits, int min_tiles, long long fit, char* part, size_t piece) {
    const long long grid = (kMost / 2) / std::max(1LL, (long long)n_tiles * p->Hkv);
    s.splits = (int)std::max<long long>(1, std::min<long long>(splits, std::min(fit, grid)));
    s.min_tiles = min_tiles;
    s.n_tiles = n_tiles;
    s.by_tiles = s2::div_by(n_tiles);
    s.by_groups = s2::div_by(p->Hkv * s.splits);
    s.by_splits = s2::div_by(s.splits);
    s.by_min = s2::div_by(min_tiles);
    s.part_rows = piece / ((p->D + 1) * sizeof(float));
    s.part_o = reinterpret_cast<float*>(part);
    return n_tiles * p->Hkv * s.splits;
  };
  a.few_rows = x.few_rows;
  a.few_tokens = x.few_tokens;
  a.by_few_tokens = s2::div_by(x.few_tokens);
  a.chunk_rows = x.chunk_rows;
  a.chunk_blocks = set(a.chunk, (int)row_tiles(p, x.chunk_rows), x.chunk_splits, x.chunk_min, fit_chunk, ws + few_bytes, y.piece);
  if (!x.chunk) a.chunk_blocks = 0;
  a.few_slots = y.slots;
  set(a.few, p->B + (p->T - 1) / x.few_tokens, x.few_splits, x.few_min, fit_few, ws, y.slots ? y.slot_piece : y.piece);
  const int splits = std::max(a.chunk.splits, a.few.splits);
  for (s2::PSet* s : {&a.chunk, &a.few})
    s->part_lse = s->part_o + (size_t)(y.slots ? s->splits : splits) * s->part_rows * p->D;   // behind all pieces of the area
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool bf16 = p->dtype == S2ATTN_BF16, e4m3 = p->cache_dtype == S2ATTN_E4M3;
  rc = bf16 ? s2::launch_paged_bf16(a, p->D, e4m3, x.nq, st) : s2::launch_paged_f32(a, p->D, e4m3, st);
  if (rc == 0 && splits > 1) rc = s2::launch_paged_join(a, p->D, bf16, x.nq, st);
  return launched(rc);
}

}  // extern "C"
