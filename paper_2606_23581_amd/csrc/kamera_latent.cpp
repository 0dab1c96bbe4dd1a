// Host side of the C ABI for serving from a paged latent cache: argument validation
// (no HIP call happens before every check has passed), translation into kernel
// parameters, launch.  The operators are defined in include/kamera.h.

#include <math.h>
#include <string.h>

#include <algorithm>

#include "kamera_host.h"
#include "kamera_latent.h"
#include "kamera_rope.h"

using namespace kamera::host;

namespace {

// A strided tensor: its rows of `width` contiguous elements.
struct View {
  const void* base;
  const int64_t* s;
  const int64_t* ext;
  int nd;
  int64_t width;
  int open = -1;                     // a dimension of which only one element is known to be there
};

bool range_of(const View& v, Range& r) { return span(v.base, v.s, v.ext, v.nd, v.width, 2, r.lo, r.hi); }

// Where the elements of a view lie within a stride `s`: in its first `in` places, counted from the base; false
// where that is not so.  Dimensions of a multiple of s leave an element's place as it is.
bool within(const View& v, int64_t s, __int128& in) {
  in = v.width;
  for (int k = 0; k < v.nd; ++k) {
    if (v.s[k] % s == 0 || (v.ext[k] <= 1 && k != v.open)) continue;
    if (v.s[k] < 0 || (k == v.open && v.s[k] > s)) return false;
    in += (__int128)(v.ext[k] - 1) * v.s[k];
  }
  return in <= s;
}

// Two views whose ranges overlap, but not their elements: the places of one within some stride lie beside those of
// the other (keys and values of a token, columns of one row).
bool beside(const View& a, const View& b) {
  const __int128 d = (__int128)(uintptr_t)b.base - (__int128)(uintptr_t)a.base;
  if (d % 2 != 0) return false;
  for (const View* v : {&a, &b})
    for (int k = 0; k < v->nd; ++k) {
      const int64_t s = v->s[k];
      __int128 in_a, in_b;
      if (s <= 0 || !within(a, s, in_a) || !within(b, s, in_b)) continue;
      const __int128 at = (d / 2 % s + s) % s;     // b's first place, a's being 0
      if (in_a <= at && at + in_b <= s) return true;
    }
  return false;
}

int check_rows(const void* p, const int64_t* s, int n, const char* what, const char* who) {
  if (!aligned16(p) || !multiples(s, n, 8))
    return fail(KAMERA_ERR_ALIGN, "%s: rows of %s must start at 16-byte boundaries", who, what);
  return KAMERA_OK;
}

// A stride in bytes (one that does not fit belongs to a dimension of one element).
int64_t in_bytes(int64_t s) { return (int64_t)((uint64_t)s * 2); }

// ---------------------------------------------------------------------------

int check_scaling(const kamera_rope_scaling& s, const char* who) {
  if (s.kind < KAMERA_SCALING_NONE || s.kind > KAMERA_SCALING_PAIRS)
    return fail(KAMERA_ERR_SHAPE, "%s: unknown scaling.kind %d", who, s.kind);
  if (!isfinite(s.amplitude)) return fail(KAMERA_ERR_SHAPE, "%s: scaling.amplitude must be finite", who);
  if (s.kind == KAMERA_SCALING_NONE) return KAMERA_OK;
  if (!(s.factor > 0.0) || !isfinite(s.factor))
    return fail(KAMERA_ERR_SHAPE, "%s: scaling.factor must be a finite positive number (got %g)", who, s.factor);
  if (s.kind == KAMERA_SCALING_LINEAR) return KAMERA_OK;
  if (!(s.original_tokens > 0.0) || !isfinite(s.original_tokens))
    return fail(KAMERA_ERR_SHAPE, "%s: scaling.original_tokens must be a finite positive number (got %g)", who,
                s.original_tokens);
  if (!(s.low_turns > 0.0) || !(s.low_turns < s.high_turns) || !isfinite(s.high_turns))
    return fail(KAMERA_ERR_SHAPE, "%s: scaling needs 0 < low_turns < high_turns (got %g, %g)", who, s.low_turns,
                s.high_turns);
  return KAMERA_OK;
}

// Scales the frequencies (revolutions a position) in place.
void scale_rope(const kamera_rope& r, const kamera_rope_scaling& s, kamera::RopeParams& o) {
  if (s.kind == KAMERA_SCALING_NONE) return;
  const int half = r.rope_dim / 2;
  double lo = 0.0, hi = 0.0;
  if (s.kind == KAMERA_SCALING_PAIRS) {
    const auto pair = [&](double turns) { return half * log(s.original_tokens / (kTwoPi * turns)) / log(r.theta); };
    lo = std::max(floor(pair(s.high_turns)), 0.0);
    hi = std::min(ceil(pair(s.low_turns)), r.rope_dim - 1.0);
  }
  for (int j = 0; j < half; ++j) {
    double keep = 0.0;
    if (s.kind == KAMERA_SCALING_TURNS)
      keep = (s.original_tokens * o.rev_freq[j] - s.low_turns) / (s.high_turns - s.low_turns);
    else if (s.kind == KAMERA_SCALING_PAIRS)
      keep = 1.0 - (j - lo) / std::max(hi - lo, 0.001);
    keep = std::min(std::max(keep, 0.0), 1.0);
    o.rev_freq[j] *= keep + (1.0 - keep) / s.factor;
  }
}

// A plane of the append: pieces of a head's row, those of the band first.
void fill_plane(kamera::RotatePlane& pl, const void* in, const int64_t* in_s, void* out, const int64_t* out_s,
                int32_t heads, int32_t dim, const kamera_rope& r, int32_t band_at) {
  pl.in = static_cast<const uint16_t*>(in);
  pl.out = static_cast<uint16_t*>(out);
  memcpy(pl.in_s, in_s, sizeof(pl.in_s));
  memcpy(pl.out_s, out_s, sizeof(pl.out_s));
  pl.n_heads = heads;
  const int band = band_at >= 0 ? r.rope_dim / 8 : 0;
  pl.band_items = r.pairing == KAMERA_PAIR_NEOX ? band / 2 : band;
  pl.band_vec = band_at >= 0 ? band_at / 8 : 0;
  pl.n_items = dim / 8 - band + pl.band_items;
  pl.fd_heads = kamera::make_fast_div((uint32_t)heads);
  pl.fd_items = kamera::make_fast_div((uint32_t)pl.n_items);
}

int build_rotate(const kamera_append_rotated_args* a, kamera::RotateParams& P, bool& launch) {
  const char* who = "kamera_append_rotated";
  launch = false;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_chunks < 0 || a->n_layers < 0 || a->n_tokens < 0 || a->n_k_heads < 0 || a->n_v_heads < 0 || a->n_q_heads < 0)
    return fail(KAMERA_ERR_SHAPE, "%s: negative n_chunks/n_layers/n_tokens/heads", who);
  const bool has_v = a->v != nullptr, has_q = a->q != nullptr;
  if (a->k_dim <= 0 || a->k_dim % 8 != 0 || (has_v && (a->v_dim <= 0 || a->v_dim % 8 != 0)))
    return fail(KAMERA_ERR_SHAPE, "%s: k_dim %d and v_dim %d must be positive multiples of 8", who, a->k_dim, a->v_dim);
  if (a->k_dim > KAMERA_MAX_HEAD_DIM || (has_v && a->v_dim > KAMERA_MAX_HEAD_DIM))
    return fail(KAMERA_ERR_RANGE, "%s: rows of more than %d columns", who, KAMERA_MAX_HEAD_DIM);
  int rc = check_rope(a->rope, a->k_dim, who);
  if (rc) return rc;
  const int need = a->rope.pairing == KAMERA_PAIR_NEOX ? 16 : 8;
  if (a->rope.rope_offset % 8 != 0 || a->rope.rope_dim % need != 0)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: rope_offset must be a multiple of 8 and rope_dim of %d", who, need);
  if ((rc = check_scaling(a->scaling, who))) return rc;
  if (a->scaling.kind == KAMERA_SCALING_PAIRS && !(a->rope.theta > 1.0))
    return fail(KAMERA_ERR_SHAPE, "%s: this scaling needs rope.theta > 1 (got %g)", who, a->rope.theta);
  if (a->page_size <= 0) return fail(KAMERA_ERR_SHAPE, "%s: page_size must be positive", who);
  if (a->n_chunks == 0 || a->n_layers == 0 || a->n_tokens == 0) return KAMERA_OK;
  const int32_t row = row_pages(a->pt_stride, a->pt_pages);
  if ((rc = check_table(a->page_table, a->pt_stride, row, a->page_size, a->n_pool_pages, 0, who))) return rc;
  if (a->k == nullptr || a->k_cache == nullptr) return fail(KAMERA_ERR_NULL, "%s: k and k_cache are needed", who);
  if (has_v != (a->v_cache != nullptr)) return fail(KAMERA_ERR_NULL, "%s: v and v_cache go together", who);
  if (has_q != (a->q_out != nullptr)) return fail(KAMERA_ERR_NULL, "%s: q and q_out go together", who);
  if (a->rope.n_sections == 3 && a->positions == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: a rope with sections needs positions", who);
  if ((rc = check_rows(a->k, a->k_stride, 4, "k", who)) || (rc = check_rows(a->k_cache, a->k_cache_stride, 4, "k_cache", who)))
    return rc;
  if (has_v && ((rc = check_rows(a->v, a->v_stride, 4, "v", who)) ||
                (rc = check_rows(a->v_cache, a->v_cache_stride, 4, "v_cache", who))))
    return rc;
  if (has_q && ((rc = check_rows(a->q, a->q_stride, 4, "q", who)) || (rc = check_rows(a->q_out, a->q_out_stride, 4, "q_out", who))))
    return rc;
  const int64_t kh = a->n_k_heads, vh = has_v ? a->n_v_heads : 0, qh = has_q ? a->n_q_heads : 0;
  if (kh * a->k_dim > 1 << 24 || vh * a->v_dim > 1 << 24 || qh * a->rope.rope_dim > 1 << 24)
    return fail(KAMERA_ERR_RANGE, "%s: more than 2^24 columns of a token", who);
  memset(&P, 0, sizeof(P));
  fill_rope(a->rope, P.rope);
  scale_rope(a->rope, a->scaling, P.rope);
  P.amplitude = a->scaling.amplitude == 0.0 ? 1.0f : (float)a->scaling.amplitude;
  if (kh > 0) fill_plane(P.plane[0], a->k, a->k_stride, a->k_cache, a->k_cache_stride, (int32_t)kh, a->k_dim, a->rope, a->rope.rope_offset);
  if (vh > 0) fill_plane(P.plane[1], a->v, a->v_stride, a->v_cache, a->v_cache_stride, (int32_t)vh, a->v_dim, a->rope, -1);
  if (qh > 0) fill_plane(P.plane[2], a->q, a->q_stride, a->q_out, a->q_out_stride, (int32_t)qh, a->rope.rope_dim, a->rope, 0);
  // what overlaps; how far rows reach is known only without a row base
  const int64_t n = a->row_base != nullptr ? 1 : a->n_tokens;
  const int64_t ext_k[4] = {a->n_chunks, a->n_layers, n, kh}, ext_v[4] = {a->n_chunks, a->n_layers, n, vh};
  const int64_t ext_q[4] = {a->n_chunks, a->n_layers, n, qh};
  const int64_t ext_kc[4] = {a->n_layers, a->n_pool_pages, a->page_size, kh};
  const int64_t ext_vc[4] = {a->n_layers, a->n_pool_pages, a->page_size, vh};
  const int open = a->row_base != nullptr ? 2 : -1;
  const View in[3] = {{a->k, a->k_stride, ext_k, 4, a->k_dim, open}, {a->v, a->v_stride, ext_v, 4, a->v_dim, open},
                      {a->q, a->q_stride, ext_q, 4, a->rope.rope_dim, open}};
  const View out[3] = {{a->k_cache, a->k_cache_stride, ext_kc, 4, a->k_dim}, {a->v_cache, a->v_cache_stride, ext_vc, 4, a->v_dim},
                       {a->q_out, a->q_out_stride, ext_q, 4, a->rope.rope_dim, open}};
  const int64_t heads[3] = {kh, vh, qh};
  Range in_r[3] = {}, out_r[3] = {};
  for (int i = 0; i < 3; ++i)
    if (heads[i] > 0 && (!range_of(in[i], in_r[i]) || !range_of(out[i], out_r[i])))
      return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  const int64_t rows = a->positions != nullptr ? n : 0;
  Range pos = {};
  const int64_t ext_p[3] = {a->n_chunks, n, a->rope.n_sections};
  if (rows > 0 && !span(a->positions, a->position_stride, ext_p, 3, 1, 4, pos.lo, pos.hi))
    return fail(KAMERA_ERR_RANGE, "%s: positions span more than the address space", who);
  const Range small[5] = {table_range(a->page_table, a->n_chunks, a->pt_stride, row), flat_or(a->chunk_tokens, a->n_chunks, 4),
                          flat_or(a->tokens_before, a->n_chunks, 4), flat_or(a->row_base, a->n_chunks, 4), pos};
  for (int o = 0; o < 3; ++o) {
    for (const Range& s : small)
      if (meet(out_r[o], s)) return fail(KAMERA_ERR_ALIAS, "%s: an output overlaps an input", who);
    for (int i = 0; i < 3; ++i) {
      if (!meet(out_r[o], in_r[i])) continue;
      const bool in_place = o == 2 && i == 2 && a->q == a->q_out && memcmp(a->q_stride, a->q_out_stride, sizeof(a->q_stride)) == 0;
      // the pool's tokens and new rows are laid out by different strides
      if (!in_place && !(o == 2 && beside(out[o], in[i])))
        return fail(KAMERA_ERR_ALIAS, "%s: an output overlaps an input", who);
    }
    for (int i = o + 1; i < 3; ++i)
      if (meet(out_r[o], out_r[i]) && !(i < 2 && beside(out[o], out[i])))
        return fail(KAMERA_ERR_ALIAS, "%s: two outputs overlap", who);
  }
  P.chunk_tokens = a->chunk_tokens;
  P.tokens_before = a->tokens_before;
  P.row_base = a->row_base;
  P.page_table = a->page_table;
  P.positions = a->positions;
  memcpy(P.position_s, a->position_stride, sizeof(P.position_s));
  P.status = a->status;
  P.n_tokens = a->n_tokens;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.pt_pages = row;
  P.n_pool_pages = a->n_pool_pages;
  P.n_layers = a->n_layers;
  // Tokens of a workgroup: about four batches of pieces a thread, fewer where that
  // leaves less than four workgroups a CU.
  int64_t items = 0;
  for (const kamera::RotatePlane& pl : P.plane) items += (int64_t)pl.n_heads * pl.n_items;
  int tb = kamera::kRotateTokens;
  while (tb > 1 && (tb * items > 4096 || (int64_t)a->n_chunks * a->n_layers * ceil_div(a->n_tokens, tb) < 1024)) tb /= 2;
  P.block_tokens = tb;
  P.n_blocks = (int32_t)ceil_div(a->n_tokens, tb);
  const int64_t tasks = bounded_product({a->n_chunks, a->n_layers, P.n_blocks});
  if (tasks < 0 || tasks * 256 > 0xFFFFFFFFLL) return fail(KAMERA_ERR_RANGE, "%s: too many tokens for one launch", who);
  P.n_tasks = (int32_t)tasks;
  P.fd_blocks = kamera::make_fast_div((uint32_t)P.n_blocks);
  P.fd_layers = kamera::make_fast_div((uint32_t)a->n_layers);
  P.fd_page = kamera::make_fast_div((uint32_t)a->page_size);
  launch = kh + vh + qh > 0;
  return KAMERA_OK;
}

// ---------------------------------------------------------------------------

// What the two products have in common: sizes, W, the tiles.
int build_product(int32_t heads, int32_t n_in, int32_t n_out, const void* w, const int64_t* w_s, int64_t requests,
                  int64_t rows, kamera::ProjectParams& P, const char* who) {
  if (w == nullptr) return fail(KAMERA_ERR_NULL, "%s: w is NULL", who);
  if (w_s[1] != 1 && w_s[2] != 1)
    return fail(KAMERA_ERR_ALIGN, "%s: the inputs or the outputs of w must be contiguous", who);
  P.w_k = w_s[2] != 1 ? 1 : 0;
  const int64_t s[2] = {w_s[0], P.w_k ? w_s[2] : w_s[1]};
  int rc = check_rows(w, s, 2, "w", who);
  if (rc) return rc;
  P.w = static_cast<const uint16_t*>(w);
  memcpy(P.w_s, w_s, sizeof(P.w_s));
  P.n_heads = heads;
  P.n_in = n_in;
  P.n_out = n_out;
  // Tiles of 32 rows for a few, which more CUs share (64 rows of 16 heads, 128 x 512: kernel 4.2 us, 5.8 in tiles of
  // 128).  Tiles of 256 need half the operands for each product, but there is one to a CU: they are taken where the
  // last round of the 256 CUs is not left mostly empty (us in tiles of 256 / 128, 16 heads, 512 x 256: 224 tiles 24.6 /
  // 28.3, 320 tiles 39.4 / 36.5, 384 tiles 40.4 / 43.5, 640 tiles 59.7 / 59.8, 1024 tiles 91 / 122; 128 tiles 19.3 / 15.0).
  P.tile_rows = rows <= 64 ? 32 : 128;
  if (n_out % 256 == 0 && rows >= 256) {
    const int64_t tiles = bounded_product({requests, ceil_div(rows, 256), heads, n_out / 256});
    if (tiles >= 1024 || (tiles >= 192 && (tiles - 1) % 256 >= 96)) P.tile_rows = 256;
  }
  P.n_row_blocks = (int32_t)ceil_div(rows, P.tile_rows);
  P.n_col_blocks = (int32_t)ceil_div(n_out, P.tile_rows == 256 ? 256 : 128);
  const int64_t tasks = bounded_product({requests, heads, P.n_row_blocks, P.n_col_blocks});
  if (tasks < 0 || (tasks + 8) * 512 > 0xFFFFFFFFLL) return fail(KAMERA_ERR_RANGE, "%s: too many tiles for one launch", who);
  P.n_tasks = (int32_t)tasks;
  P.per_xcd = (int32_t)ceil_div(tasks, 8);
  P.fd_rows = kamera::make_fast_div((uint32_t)P.n_row_blocks);
  P.fd_cols = kamera::make_fast_div((uint32_t)P.n_col_blocks);
  P.fd_heads = kamera::make_fast_div((uint32_t)heads);
  return KAMERA_OK;
}

int check_product_sizes(int32_t heads, int32_t n_in, int32_t n_out, const char* who) {
  if (heads < 0) return fail(KAMERA_ERR_SHAPE, "%s: negative n_heads", who);
  if (n_in <= 0 || n_out <= 0 || n_in % 64 != 0 || n_out % 64 != 0)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: n_in %d and n_out %d must be multiples of 64", who, n_in, n_out);
  if (n_in > KAMERA_MAX_HEAD_DIM || n_out > KAMERA_MAX_HEAD_DIM)
    return fail(KAMERA_ERR_RANGE, "%s: more than %d columns", who, KAMERA_MAX_HEAD_DIM);
  return KAMERA_OK;
}

int build_project(const kamera_project_args* a, kamera::ProjectParams& P, bool& launch) {
  const char* who = "kamera_project_heads";
  launch = false;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_rows < 0) return fail(KAMERA_ERR_SHAPE, "%s: negative n_rows", who);
  int rc = check_product_sizes(a->n_heads, a->n_in, a->n_out, who);
  if (rc) return rc;
  if (a->n_rows == 0 || a->n_heads == 0) return KAMERA_OK;
  if (a->x == nullptr || a->out == nullptr) return fail(KAMERA_ERR_NULL, "%s: x, w and out are needed", who);
  memset(&P, 0, sizeof(P));
  if ((rc = build_product(a->n_heads, a->n_in, a->n_out, a->w, a->w_stride, 1, a->n_rows, P, who))) return rc;
  if ((rc = check_rows(a->x, a->x_stride, 2, "x", who)) || (rc = check_rows(a->out, a->out_stride, 2, "out", who))) return rc;
  const int64_t ext[2] = {a->n_rows, a->n_heads}, ext_w[3] = {a->n_heads, a->n_in, a->n_out};
  const View x = {a->x, a->x_stride, ext, 2, a->n_in}, out = {a->out, a->out_stride, ext, 2, a->n_out};
  Range xr, wr, o;
  if (!range_of(x, xr) || !range_of(out, o) || !span(a->w, a->w_stride, ext_w, 3, 1, 2, wr.lo, wr.hi))
    return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  if (meet(o, wr) || (meet(o, xr) && !beside(out, x))) return fail(KAMERA_ERR_ALIAS, "%s: out overlaps an input", who);
  P.x = static_cast<const uint16_t*>(a->x);
  P.out = static_cast<uint16_t*>(a->out);
  memcpy(P.x_s, a->x_stride, sizeof(P.x_s));
  memcpy(P.out_s, a->out_stride, sizeof(P.out_s));
  P.n_rows = a->n_rows;
  P.n_requests = 1;
  P.fd_page = kamera::make_fast_div(1);
  launch = true;
  return KAMERA_OK;
}

int build_expand(const kamera_expand_args* a, kamera::ProjectParams& P, bool& launch) {
  const char* who = "kamera_expand_latent";
  launch = false;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_requests < 0 || a->n_keys < 0) return fail(KAMERA_ERR_SHAPE, "%s: negative n_requests/n_keys", who);
  int rc = check_product_sizes(a->n_heads, a->n_in, a->n_out, who);
  if (rc) return rc;
  if (a->page_size <= 0) return fail(KAMERA_ERR_SHAPE, "%s: page_size must be positive", who);
  if (a->n_requests == 0 || a->n_heads == 0 || a->n_keys == 0) return KAMERA_OK;
  if ((rc = check_table(a->page_table, a->pt_stride, a->pt_stride, a->page_size, a->n_pool_pages, a->n_keys, who))) return rc;
  if (a->kv_tokens == nullptr || a->cache == nullptr || a->out == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: kv_tokens, cache, w and out are needed", who);
  memset(&P, 0, sizeof(P));
  if ((rc = build_product(a->n_heads, a->n_in, a->n_out, a->w, a->w_stride, a->n_requests, a->n_keys, P, who))) return rc;
  if ((rc = check_rows(a->cache, a->cache_stride, 2, "cache", who)) || (rc = check_rows(a->out, a->out_stride, 2, "out", who)))
    return rc;
  // how far out reaches is known only without a row base
  const int64_t rows = a->row_base != nullptr ? 1 : bounded_product({a->n_requests, a->n_keys});
  if (rows < 0) return fail(KAMERA_ERR_RANGE, "%s: too many rows", who);
  const int64_t ext[2] = {rows, a->n_heads}, ext_c[2] = {a->n_pool_pages, a->page_size};
  const int64_t ext_w[3] = {a->n_heads, a->n_in, a->n_out};
  Range in[5], o;
  if (!span(a->cache, a->cache_stride, ext_c, 2, a->n_in, 2, in[0].lo, in[0].hi) ||
      !span(a->w, a->w_stride, ext_w, 3, 1, 2, in[1].lo, in[1].hi) ||
      !span(a->out, a->out_stride, ext, 2, a->n_out, 2, o.lo, o.hi))
    return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  in[2] = table_range(a->page_table, a->n_requests, a->pt_stride, (int32_t)ceil_div(a->n_keys, a->page_size));
  in[3] = flat(a->kv_tokens, a->n_requests, 4);
  in[4] = flat_or(a->row_base, a->n_requests, 4);
  for (const Range& r : in)
    if (meet(o, r)) return fail(KAMERA_ERR_ALIAS, "%s: out overlaps an input", who);
  P.x = static_cast<const uint16_t*>(a->cache);
  P.out = static_cast<uint16_t*>(a->out);
  memcpy(P.x_s, a->cache_stride, sizeof(P.x_s));
  memcpy(P.out_s, a->out_stride, sizeof(P.out_s));
  P.paged = 1;
  P.kv_tokens = a->kv_tokens;
  P.row_base = a->row_base;
  P.page_table = a->page_table;
  P.status = a->status;
  P.n_requests = a->n_requests;
  P.n_keys = a->n_keys;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.n_pool_pages = a->n_pool_pages;
  P.fd_page = kamera::make_fast_div((uint32_t)a->page_size);
  launch = true;
  return KAMERA_OK;
}

// ---------------------------------------------------------------------------

// What the two forms of attention take alike.
struct AttendSizes {
  int32_t n_requests, n_heads, dim, n_queries, n_keys, page_size, causal, window, n_parts;
  float scale;
  bool latent;
};

// Sizes of a call, and how its work is divided.
int size_mla(const AttendSizes& a, kamera::MlaParams& P, bool& launch, int64_t& workspace, const char* who) {
  launch = false;
  workspace = 0;
  if (a.n_requests < 0 || a.n_queries < 0 || a.n_keys < 0)
    return fail(KAMERA_ERR_SHAPE, "%s: negative n_requests/n_queries/n_keys", who);
  if (a.n_heads <= 0) return fail(KAMERA_ERR_SHAPE, "%s: n_heads must be positive (got %d)", who, a.n_heads);
  if (a.page_size <= 0 || a.page_size % 16 != 0)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: page_size must be a multiple of 16 (got %d)", who, a.page_size);
  if (a.causal != 0 && a.causal != 1) return fail(KAMERA_ERR_SHAPE, "%s: causal must be 0 or 1", who);
  if (a.window < 0 || (a.window > 0 && !a.causal))
    return fail(KAMERA_ERR_SHAPE, "%s: a window must be positive and needs causal = 1", who);
  if (!isfinite(a.scale)) return fail(KAMERA_ERR_SHAPE, "%s: scale must be finite", who);
  if (a.n_parts < 0 || a.n_parts > 1024) return fail(KAMERA_ERR_SHAPE, "%s: n_parts must be 0 .. 1024", who);
  // token positions, and those of the tile after the last one, stay in 31 bits
  if ((int64_t)a.n_keys + a.n_queries > INT32_MAX - 4096)
    return fail(KAMERA_ERR_RANGE, "%s: too many keys or queries a request", who);
  if (a.n_requests == 0 || a.n_queries == 0) return KAMERA_OK;
  memset(&P, 0, sizeof(P));
  P.group = a.latent ? a.n_heads : 1;
  P.task_heads = a.latent ? 1 : a.n_heads;
  const int64_t rows = (int64_t)a.n_queries * P.group;
  if (rows > INT32_MAX / 2) return fail(KAMERA_ERR_RANGE, "%s: too many query rows", who);
  // the fewest waves that have all rows of a request, from 33 rows on 8, whose keys are fetched once for 128 rows
  // (64 requests of up to 8192 keys: 24 heads 90.4 us with 2, 93.0 with 8; 48 heads 102.5 with 8, 103.8 with two
  // groups of 4, 137 with 2)
  P.row_waves = rows > 32 ? 8 : (rows > 16 ? 2 : 1);
  P.rows_block = a.latent ? 16 * P.row_waves : 128;
  P.n_row_blocks = (int32_t)ceil_div(rows, P.rows_block);
  const int64_t tasks = bounded_product({a.n_requests, P.task_heads, P.n_row_blocks});
  const int threads = a.latent ? kamera::latent_waves(P.row_waves) * 64 : 256;
  if (tasks < 0 || (tasks + 8) * threads > 0xFFFFFFFFLL) return fail(KAMERA_ERR_RANGE, "%s: too many workgroups for one launch", who);
  P.n_tasks = (int32_t)tasks;
  const int unit = P.unit = a.latent ? 32 * kamera::latent_groups(P.row_waves) : 64;
  // what 256 keys cost, 288 of the latent form's blocks of 128 rows (us with none of it, half of it, all, half as much
  // again: eight ragged prompts, expanded, 143, 123, 115, 116; 64 single queries of 16 heads, latent, 91.0, 89.3, 87.8,
  // 88.0; 16 requests of two queries of 128 heads 90 with 128 keys, 87.4 with 192, 85.3 with 288, 86.2 with 384)
  P.fixed = (a.latent ? 288 : 256) / unit;
  P.lanes = 1;
  while (P.lanes < 64 && P.lanes < P.n_row_blocks) P.lanes *= 2;
  int64_t keys = a.n_keys;
  if (a.window > 0) keys = std::min<int64_t>(keys, (int64_t)a.window + a.n_queries);
  const int64_t units = keys / unit + 2, total = bounded_product({tasks, units + P.fixed});
  const bool can = total >= 0 && total <= INT32_MAX / 2;
  if (a.n_parts > 0) {
    if (!can) return fail(KAMERA_ERR_RANGE, "%s: too much work to divide", who);
    P.n_parts = a.n_parts;
    P.min_units = 1;
  } else if (can && tasks < kamera::kMlaDivideTasks && units > (a.latent ? 6 : 10)) {
    // Up to 512 keys (latent, 16 rows; expanded) one workgroup is done before a second could have joined its part.  One
    // request, us whole / divided: single query of 16 heads, 512 keys 15.4 / 17.3, 640 17.1 / 17.6, 768 18.8 / 17.5;
    // 128 queries of 16 heads, expanded, 512 keys 20.8 / 20.3, 576 22.2 / 20.7, 1024 31.9 / 22.3.  Blocks of more rows
    // have shorter units and are divided from fewer keys on: 32 rows, 256 keys 14.0 / 18.1, 320 15.5 / 18.4, 448 18.2 /
    // 18.5, 512 19.6 / 18.4; 128 rows, 128 keys 22.4 / 25.2, 192 25.9 / 25.5, 256 29.4 / 25.4.  Many requests would gain
    // from later on: 16 of 128 rows, 192 keys 26.6 / 32.7, 320 33.7 / 33.2; 64 of them, 192 keys 27.7 / 41.8, 512
    // 46.0 / 48.6.  A part is 128 keys of the latent form, which its four groups take at once, else two units (single
    // queries of 128 heads, 256 keys: 26.2 us, 27.8 in parts of one).
    P.min_units = unit == 128 ? 1 : 2;
    P.n_parts = (int32_t)std::min<int64_t>(a.latent ? 256 : 512, ceil_div(total, P.min_units));
  }
  if (P.n_parts > 0) {
    workspace = bounded_product({P.n_parts, 2, P.rows_block, a.dim + 4, 4});
    if (workspace < 0) return fail(KAMERA_ERR_RANGE, "%s: workspace too large", who);
    workspace += ceil_div((tasks + 1 + P.n_parts) * 4, 16) * 16;
  }
  launch = true;
  return KAMERA_OK;
}

template <typename A>
AttendSizes sizes_of(const A* a, int32_t dim, bool latent) {
  return {a->n_requests, a->n_heads, dim, a->n_queries, a->n_keys, a->page_size, a->causal, a->window, a->n_parts, a->scale, latent};
}

int size_latent(const kamera_attend_latent_args* a, kamera::MlaParams& P, bool& launch, int64_t& workspace) {
  const char* who = "kamera_attend_latent";
  launch = false;
  workspace = 0;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if ((a->latent_dim != 256 && a->latent_dim != 512) || a->rope_dim != kamera::kRopeCols)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: latent_dim must be 256 or 512 and rope_dim 64 (got %d, %d)", who, a->latent_dim,
                a->rope_dim);
  return size_mla(sizes_of(a, a->latent_dim, true), P, launch, workspace, who);
}

int size_expanded(const kamera_attend_expanded_args* a, kamera::MlaParams& P, bool& launch, int64_t& workspace) {
  const char* who = "kamera_attend_expanded";
  launch = false;
  workspace = 0;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if ((a->head_dim != 64 && a->head_dim != 128) || a->rope_dim != kamera::kRopeCols)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 and rope_dim 64 (got %d, %d)", who, a->head_dim,
                a->rope_dim);
  return size_mla(sizes_of(a, a->head_dim, false), P, launch, workspace, who);
}

// Checks, ranges and parameters of what both take: q, out, lse, page table, pool, workspace.
// in[0 .. n_in) are filled by the caller; six more are added.
template <typename A>
int build_mla(const A* a, int32_t dim, const void* pool, const int64_t* pool_s, int32_t pool_cols, Range* in, int n_in,
              int64_t workspace, kamera::MlaParams& P, const char* who) {
  int rc = check_table(a->page_table, a->pt_stride, a->pt_stride, a->page_size, a->n_pool_pages, a->n_keys, who);
  if (rc) return rc;
  if (a->kv_tokens == nullptr || a->q == nullptr || a->out == nullptr || pool == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: kv_tokens, q, out and the cache are needed", who);
  if ((rc = check_rows(a->q, a->q_stride, 2, "q", who)) || (rc = check_rows(a->out, a->out_stride, 2, "out", who)) ||
      (rc = check_rows(pool, pool_s, 2, "the cache", who)))
    return rc;
  // lane offsets within a tile are 32-bit
  if (pool_s[1] < 0 || pool_s[1] > (int64_t)1 << 24)
    return fail(KAMERA_ERR_RANGE, "%s: token stride %lld of the cache", who, (long long)pool_s[1]);
  // how far rows reach is known only without a row base
  const int64_t n_rows = a->q_base != nullptr ? 1 : (int64_t)a->n_requests * a->n_queries;
  const int64_t ext_q[2] = {n_rows, a->n_heads}, ext_p[2] = {a->n_pool_pages, a->page_size};
  Range out[3] = {};
  if (!span(a->q, a->q_stride, ext_q, 2, dim + a->rope_dim, 2, in[n_in].lo, in[n_in].hi) ||
      !span(pool, pool_s, ext_p, 2, pool_cols, 2, in[n_in + 1].lo, in[n_in + 1].hi) ||
      !span(a->out, a->out_stride, ext_q, 2, dim, 2, out[0].lo, out[0].hi) ||
      (a->lse != nullptr && !span(a->lse, a->lse_stride, ext_q, 2, 1, 4, out[1].lo, out[1].hi)))
    return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  in[n_in + 2] = table_range(a->page_table, a->n_requests, a->pt_stride, (int32_t)ceil_div(a->n_keys, a->page_size));
  in[n_in + 3] = flat(a->kv_tokens, a->n_requests, 4);
  in[n_in + 4] = flat_or(a->q_tokens, a->n_requests, 4);
  in[n_in + 5] = flat_or(a->q_base, a->n_requests, 4);
  if (workspace > 0) {
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, workspace, who))) return rc;
    out[2] = flat(a->workspace, workspace, 1);
  }
  for (int i = 0; i < 3; ++i) {
    for (int k = 0; k < n_in + 6; ++k)
      if (meet(out[i], in[k])) return fail(KAMERA_ERR_ALIAS, "%s: out, lse or workspace overlaps an input", who);
    for (int k = i + 1; k < 3; ++k)
      if (meet(out[i], out[k])) return fail(KAMERA_ERR_ALIAS, "%s: out, lse and workspace overlap", who);
  }
  P.q_tokens = a->q_tokens;
  P.q_base = a->q_base;
  P.kv_tokens = a->kv_tokens;
  P.page_table = a->page_table;
  P.q = static_cast<const uint16_t*>(a->q);
  P.out = static_cast<uint16_t*>(a->out);
  P.lse = a->lse;
  P.pool = static_cast<const uint8_t*>(pool);
  P.status = a->status;
  for (int k = 0; k < 2; ++k) {
    P.q_s[k] = a->q_stride[k];
    P.out_s[k] = a->out_stride[k];
    P.lse_s[k] = a->lse_stride[k];
    P.pool_s[k] = in_bytes(pool_s[k]);
  }
  // the kernels take a largest score by its product with a positive factor; a
  // zero scale becomes one that leaves every score a difference of zero
  P.scale2 = std::max((float)(fabs((double)a->scale) * 1.4426950408889634074), 1e-30f);
  P.q_sign = a->scale < 0.f ? 0x80008000u : 0u;
  P.n_requests = a->n_requests;
  P.n_heads = a->n_heads;
  P.dim = dim;
  P.n_queries = a->n_queries;
  P.n_keys = a->n_keys;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.n_pool_pages = a->n_pool_pages;
  P.causal = a->causal;
  P.window = std::min(a->window, std::max(a->n_keys, 1));   // a longer one sees no more, and positions less it could wrap
  if (workspace > 0) {
    const int64_t rows = (int64_t)P.n_parts * 2 * P.rows_block;
    P.part_o = static_cast<float*>(a->workspace);
    P.part_ml = P.part_o + rows * dim;
    P.prefix = reinterpret_cast<int32_t*>(P.part_ml + rows * 4);
  }
  P.fd_group = kamera::make_fast_div((uint32_t)P.group);
  P.fd_blocks = kamera::make_fast_div((uint32_t)P.n_row_blocks);
  P.fd_heads = kamera::make_fast_div((uint32_t)P.task_heads);
  P.fd_page16 = kamera::make_fast_div((uint32_t)a->page_size / 16);
  return KAMERA_OK;
}

int build_latent(const kamera_attend_latent_args* a, kamera::MlaParams& P, bool& launch) {
  int64_t workspace = 0;
  int rc = size_latent(a, P, launch, workspace);
  if (rc || !launch) return rc;
  launch = false;
  Range in[6] = {};
  if ((rc = build_mla(a, a->latent_dim, a->cache, a->cache_stride, a->latent_dim + a->rope_dim, in, 0, workspace, P,
                      "kamera_attend_latent")))
    return rc;
  launch = true;
  return KAMERA_OK;
}

int build_expanded(const kamera_attend_expanded_args* a, kamera::MlaParams& P, bool& launch) {
  const char* who = "kamera_attend_expanded";
  int64_t workspace = 0;
  int rc = size_expanded(a, P, launch, workspace);
  if (rc || !launch) return rc;
  launch = false;
  if (a->k == nullptr || a->v == nullptr) return fail(KAMERA_ERR_NULL, "%s: k and v are needed", who);
  if ((rc = check_rows(a->k, a->k_stride, 2, "k", who)) || (rc = check_rows(a->v, a->v_stride, 2, "v", who))) return rc;
  for (const int64_t t : {a->k_stride[0], a->v_stride[0]})
    if (t < 0 || t > (int64_t)1 << 24) return fail(KAMERA_ERR_RANGE, "%s: row stride %lld of k or v", who, (long long)t);
  Range in[9] = {};
  // how far k and v reach is known only without a row base
  const int64_t rows = a->kv_base != nullptr ? 1 : (int64_t)a->n_requests * a->n_keys;
  const int64_t ext[2] = {rows, a->n_heads};
  if (!span(a->k, a->k_stride, ext, 2, a->head_dim, 2, in[0].lo, in[0].hi) ||
      !span(a->v, a->v_stride, ext, 2, a->head_dim, 2, in[1].lo, in[1].hi))
    return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  in[2] = flat_or(a->kv_base, a->n_requests, 4);
  if ((rc = build_mla(a, a->head_dim, a->rope_cache, a->rope_cache_stride, a->rope_dim, in, 3, workspace, P, who))) return rc;
  P.k = static_cast<const uint8_t*>(a->k);
  P.v = static_cast<const uint8_t*>(a->v);
  P.kv_base = a->kv_base;
  for (int k = 0; k < 2; ++k) {
    P.k_s[k] = in_bytes(a->k_stride[k]);
    P.v_s[k] = in_bytes(a->v_stride[k]);
  }
  launch = true;
  return KAMERA_OK;
}

int finish(hipError_t e, const char* who) {
  if (e != hipSuccess) return fail(KAMERA_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ok();
}

// Builds a call's parameters and launches it.
template <typename Params, typename Args>
int run(const Args* a, void* stream, int (*build)(const Args*, Params&, bool&), hipError_t (*launch)(const Params&, hipStream_t),
        const char* who) {
  Params P;
  bool there = false;
  const int rc = build(a, P, there);
  if (rc) return rc;
  return finish(there ? launch(P, static_cast<hipStream_t>(stream)) : hipSuccess, who);
}

template <typename Params, typename Args>
int check(const void* a, int (*build)(const Args*, Params&, bool&)) {
  Params P;
  bool there = false;
  const int rc = build(static_cast<const Args*>(a), P, there);
  return rc ? rc : ok();
}

}  // namespace

extern "C" int kamera_append_rotated(const kamera_append_rotated_args* a, void* stream) {
  return run(a, stream, build_rotate, kamera::launch_rotate, "kamera_append_rotated");
}

extern "C" int kamera_project_heads(const kamera_project_args* a, void* stream) {
  return run(a, stream, build_project, kamera::launch_project, "kamera_project_heads");
}

extern "C" int kamera_expand_latent(const kamera_expand_args* a, void* stream) {
  return run(a, stream, build_expand, kamera::launch_project, "kamera_expand_latent");
}

extern "C" int kamera_attend_latent(const kamera_attend_latent_args* a, void* stream) {
  return run(a, stream, build_latent, kamera::launch_attend_latent, "kamera_attend_latent");
}

extern "C" int kamera_attend_expanded(const kamera_attend_expanded_args* a, void* stream) {
  return run(a, stream, build_expanded, kamera::launch_attend_expanded, "kamera_attend_expanded");
}

extern "C" int64_t kamera_attend_latent_workspace(const kamera_attend_latent_args* a) {
  kamera::MlaParams P;
  bool launch = false;
  int64_t workspace = 0;
  const int rc = size_latent(a, P, launch, workspace);
  if (rc) return rc;
  ok();
  return workspace;
}

extern "C" int64_t kamera_attend_expanded_workspace(const kamera_attend_expanded_args* a) {
  kamera::MlaParams P;
  bool launch = false;
  int64_t workspace = 0;
  const int rc = size_expanded(a, P, launch, workspace);
  if (rc) return rc;
  ok();
  return workspace;
}

extern "C" int kamera_validate_latent(int32_t which, const void* args) {
  switch (which) {
    case 0: return check(args, build_rotate);
    case 1: return check(args, build_project);
    case 2: return check(args, build_expand);
    case 3: return check(args, build_latent);
    case 4: return check(args, build_expanded);
    default: return fail(KAMERA_ERR_SHAPE, "kamera_validate_latent: unknown entry point %d", which);
  }
}
