// Host side of the C ABI for serving from the paged cache: argument validation
// (no HIP call happens before every check has passed), translation into kernel
// parameters, launch.  The operators are defined in include/kamera.h.

#include <math.h>
#include <string.h>

#include <algorithm>

#include "kamera_cache.h"
#include "kamera_host.h"

using namespace kamera::host;

namespace {

struct Range {
  uintptr_t lo, hi;
};

// Byte range of n elements from p.
Range flat(const void* p, int64_t n, int bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return {a, a + (uintptr_t)n * bytes};
}

// The same of an optional array.
Range flat_or(const void* p, int64_t n, int bytes) { return flat(p, p != nullptr ? n : 0, bytes); }

bool meet(const Range& a, const Range& b) { return a.lo < a.hi && b.lo < b.hi && overlap(a.lo, a.hi, b.lo, b.hi); }

bool multiples(const int64_t* s, int n, int64_t of) {
  for (int k = 0; k < n; ++k)
    if (s[k] % of != 0) return false;
  return true;
}

// Page selection: from so many pages a request on they are scored by workgroups of
// their own (see kamera_select.hip).
constexpr int64_t kSelectSplit = 1024;

int check_head_dim(int32_t head_dim, const char* who) {
  if (head_dim != 64 && head_dim != 128)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 (got %d)", who, head_dim);
  return KAMERA_OK;
}

int check_heads(int32_t q_heads, int32_t kv_heads, const char* who) {
  if (kv_heads <= 0 || q_heads <= 0 || q_heads % kv_heads != 0)
    return fail(KAMERA_ERR_SHAPE, "%s: n_q_heads %d must be a positive multiple of n_kv_heads %d", who, q_heads, kv_heads);
  if (q_heads / kv_heads > KAMERA_MAX_GROUP)
    return fail(KAMERA_ERR_RANGE, "%s: %d query heads share a KV head, at most %d can", who, q_heads / kv_heads,
                KAMERA_MAX_GROUP);
  return KAMERA_OK;
}

// `pages`: the entries of a row.
int check_table(const int32_t* table, int32_t pt_stride, int32_t pages, int32_t page_size, int32_t n_pool_pages,
                int64_t tokens, const char* who) {
  if (table == nullptr) return fail(KAMERA_ERR_NULL, "%s: page_table is NULL", who);
  if (n_pool_pages <= 0) return fail(KAMERA_ERR_SHAPE, "%s: n_pool_pages must be positive", who);
  if (pt_stride < 0 || pages < ceil_div(tokens, page_size))
    return fail(KAMERA_ERR_SHAPE, "%s: %d pages a row (stride %d) < %lld pages needed for %lld tokens", who, pages,
                pt_stride, (long long)ceil_div(tokens, page_size), (long long)tokens);
  return KAMERA_OK;
}

// Entries that a row of a page table has.
int32_t row_pages(int32_t pt_stride, int32_t pt_pages) { return pt_pages != 0 ? pt_pages : pt_stride; }

// Bytes of a table of n rows.
Range table_range(const int32_t* table, int64_t n, int32_t pt_stride, int32_t pages) {
  return flat(table, n > 0 && pages > 0 ? (n - 1) * pt_stride + pages : 0, 4);
}

int check_workspace(const void* workspace, int64_t bytes, int64_t needed, const char* who) {
  if (workspace == nullptr) return fail(KAMERA_ERR_NULL, "%s: workspace is NULL", who);
  if (bytes < needed)
    return fail(KAMERA_ERR_SHAPE, "%s: workspace of %lld bytes, %lld needed", who, (long long)bytes, (long long)needed);
  if (!aligned16(workspace)) return fail(KAMERA_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  return KAMERA_OK;
}

int check_page8(int32_t page_size, const char* who) {
  if (page_size != 16 && page_size != 32 && page_size != 64)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: pages of the 8-bit cache hold 16, 32 or 64 tokens (got %d)", who, page_size);
  return KAMERA_OK;
}

// ---------------------------------------------------------------------------

int build_tables(const kamera_page_tables_args* a, kamera::TablesParams& P, bool& launch) {
  const char* who = "kamera_page_tables";
  launch = false;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_requests < 0 || a->n_free < 0 || a->n_slots < 0)
    return fail(KAMERA_ERR_SHAPE, "%s: negative n_requests/n_free/n_slots", who);
  if (a->n_requests > KAMERA_MAX_REQUESTS)
    return fail(KAMERA_ERR_RANGE, "%s: %d requests exceed %d", who, a->n_requests, KAMERA_MAX_REQUESTS);
  if (a->page_size <= 0 || a->pt_stride <= 0 || a->n_pool_pages <= 0)
    return fail(KAMERA_ERR_SHAPE, "%s: page_size, pt_stride and n_pool_pages must be positive", who);
  const int64_t most = bounded_product({std::max(a->n_requests, 1), a->pt_stride, a->page_size});
  if (most < 0 || most > INT32_MAX)
    return fail(KAMERA_ERR_RANGE, "%s: n_requests * pt_stride * page_size must be below 2^31", who);
  if (a->n_slots > kMaxWork) return fail(KAMERA_ERR_RANGE, "%s: n_slots too large", who);
  if (a->n_requests > 0 && (a->tokens_after == nullptr || a->page_table == nullptr))
    return fail(KAMERA_ERR_NULL, "%s: tokens_after and page_table are needed", who);
  if (a->token_base == nullptr || a->free_end == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: token_base and free_end are needed", who);
  if (a->n_free > 0 && a->free_pages == nullptr) return fail(KAMERA_ERR_NULL, "%s: free_pages is NULL", who);
  if (a->n_slots > 0 && a->slots == nullptr) return fail(KAMERA_ERR_NULL, "%s: slots is NULL", who);
  const int64_t n = a->n_requests;
  const Range outs[4] = {flat(a->page_table, n * a->pt_stride, 4), flat(a->token_base, n + 1, 4),
                         flat(a->free_end, 1, 4), flat_or(a->slots, a->n_slots, 8)};
  const Range ins[4] = {flat_or(a->tokens_before, n, 4), flat(a->tokens_after, n, 4),
                        flat(a->free_pages, a->n_free, 4), flat_or(a->free_begin, 1, 4)};
  for (int i = 0; i < 4; ++i) {
    for (int k = 0; k < 4; ++k)
      if (meet(outs[i], ins[k])) return fail(KAMERA_ERR_ALIAS, "%s: an output overlaps an input", who);
    for (int k = i + 1; k < 4; ++k)
      if (meet(outs[i], outs[k])) return fail(KAMERA_ERR_ALIAS, "%s: two outputs overlap", who);
  }
  memset(&P, 0, sizeof(P));
  P.tokens_before = a->tokens_before;
  P.tokens_after = a->tokens_after;
  P.free_pages = a->free_pages;
  P.free_begin = a->free_begin;
  P.free_end = a->free_end;
  P.page_table = a->page_table;
  P.token_base = a->token_base;
  P.slots = a->n_slots > 0 ? a->slots : nullptr;
  P.n_slots = a->n_slots;
  P.slots_aligned = aligned16(a->slots) ? 1 : 0;
  P.status = a->status;
  P.n_requests = a->n_requests;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.n_pool_pages = a->n_pool_pages;
  P.n_free = a->n_free;
  P.fd_page = kamera::make_fast_div((uint32_t)a->page_size);
  launch = true;
  return KAMERA_OK;
}

// ---------------------------------------------------------------------------

int build_append(const kamera_append_args* a, kamera::AppendParams& P, bool& launch) {
  const char* who = "kamera_append_paged8";
  launch = false;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_chunks < 0 || a->n_layers < 0 || a->n_heads < 0 || a->n_tokens < 0)
    return fail(KAMERA_ERR_SHAPE, "%s: negative n_chunks/n_layers/n_heads/n_tokens", who);
  int rc = check_head_dim(a->head_dim, who);
  if (rc) return rc;
  if ((rc = check_page8(a->page_size, who))) return rc;
  if (a->n_chunks == 0 || a->n_layers == 0 || a->n_heads == 0 || a->n_tokens == 0) return KAMERA_OK;
  const int32_t row = row_pages(a->pt_stride, a->pt_pages);
  if ((rc = check_table(a->page_table, a->pt_stride, row, a->page_size, a->n_pool_pages, a->n_tokens, who))) return rc;
  if (a->k == nullptr || a->v == nullptr || a->k_cache == nullptr || a->v_cache == nullptr || a->k_scale == nullptr ||
      a->v_scale == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: k, v, their caches and scales are needed", who);
  if ((a->k_sum == nullptr) != (a->k_sum_scale == nullptr))
    return fail(KAMERA_ERR_NULL, "%s: k_sum and k_sum_scale go together", who);
  if (!aligned16(a->k) || !aligned16(a->v) || !multiples(a->k_stride, 4, 8) || !multiples(a->v_stride, 4, 8))
    return fail(KAMERA_ERR_ALIGN, "%s: rows must start at 16-byte boundaries", who);
  if (!aligned16(a->k_cache) || !aligned16(a->v_cache) || !multiples(a->k_cache_stride, 4, 16) ||
      !multiples(a->v_cache_stride, 4, 16))
    return fail(KAMERA_ERR_ALIGN, "%s: cache rows must start at 16-byte boundaries", who);
  if (a->k_sum != nullptr && (!aligned16(a->k_sum) || !multiples(a->k_sum_stride, 3, 16)))
    return fail(KAMERA_ERR_ALIGN, "%s: key sums must start at 16-byte boundaries", who);
  // the page that holds the first new token may hold page_size - 1 others
  const int64_t pages = ((int64_t)a->n_tokens + a->page_size - 2) / a->page_size + 1;
  const int64_t units = bounded_product({a->n_chunks, a->n_layers, a->n_heads, 2, pages});
  if (units < 0 || ceil_div(units, kamera::append_units_wg(a->page_size)) * kamera::kAppendThreads > 0xFFFFFFFFLL)
    return fail(KAMERA_ERR_RANGE, "%s: too many (chunk, layer, page, head) units for one launch", who);
  const int64_t ext[4] = {a->n_layers, a->n_pool_pages, a->page_size, a->n_heads};
  const int64_t ext_s[3] = {a->n_layers, a->n_pool_pages, a->n_heads};
  Range out[6] = {};
  if (!span(a->k_cache, a->k_cache_stride, ext, 4, a->head_dim, 1, out[0].lo, out[0].hi) ||
      !span(a->v_cache, a->v_cache_stride, ext, 4, a->head_dim, 1, out[1].lo, out[1].hi) ||
      !span(a->k_scale, a->k_scale_stride, ext_s, 3, 1, 4, out[2].lo, out[2].hi) ||
      !span(a->v_scale, a->v_scale_stride, ext_s, 3, 1, 4, out[3].lo, out[3].hi))
    return fail(KAMERA_ERR_RANGE, "%s: cache strides span more than the address space", who);
  if (a->k_sum != nullptr && (!span(a->k_sum, a->k_sum_stride, ext_s, 3, a->head_dim, 1, out[4].lo, out[4].hi) ||
                              !span(a->k_sum_scale, a->k_sum_scale_stride, ext_s, 3, 1, 4, out[5].lo, out[5].hi)))
    return fail(KAMERA_ERR_RANGE, "%s: k_sum strides span more than the address space", who);
  // how far the rows reach is known only without a row base
  const int64_t ext_in[4] = {a->n_chunks, a->n_layers, a->row_base != nullptr ? 1 : a->n_tokens, a->n_heads};
  Range in[6];
  if (!span(a->k, a->k_stride, ext_in, 4, a->head_dim, 2, in[0].lo, in[0].hi) ||
      !span(a->v, a->v_stride, ext_in, 4, a->head_dim, 2, in[1].lo, in[1].hi))
    return fail(KAMERA_ERR_RANGE, "%s: row strides span more than the address space", who);
  in[2] = table_range(a->page_table, a->n_chunks, a->pt_stride, row);
  in[3] = flat_or(a->chunk_tokens, a->n_chunks, 4);
  in[4] = flat_or(a->tokens_before, a->n_chunks, 4);
  in[5] = flat_or(a->row_base, a->n_chunks, 4);
  for (const Range& o : out)
    for (const Range& r : in)
      if (meet(o, r)) return fail(KAMERA_ERR_ALIAS, "%s: an output overlaps an input", who);
  if (a->k_cache == a->v_cache || a->k_scale == a->v_scale)
    return fail(KAMERA_ERR_ALIAS, "%s: keys and values need a cache each", who);
  memset(&P, 0, sizeof(P));
  const void* rows[2] = {a->k, a->v};
  void* cache[2] = {a->k_cache, a->v_cache};
  float* scale[2] = {a->k_scale, a->v_scale};
  const int64_t* rs[2] = {a->k_stride, a->v_stride};
  const int64_t* cs[2] = {a->k_cache_stride, a->v_cache_stride};
  const int64_t* ss[2] = {a->k_scale_stride, a->v_scale_stride};
  for (int pl = 0; pl < 2; ++pl) {
    P.plane[pl].rows = static_cast<const uint16_t*>(rows[pl]);
    P.plane[pl].cache = static_cast<uint8_t*>(cache[pl]);
    P.plane[pl].scale = scale[pl];
    memcpy(P.plane[pl].rows_s, rs[pl], sizeof(P.plane[pl].rows_s));
    memcpy(P.plane[pl].cache_s, cs[pl], sizeof(P.plane[pl].cache_s));
    memcpy(P.plane[pl].scale_s, ss[pl], sizeof(P.plane[pl].scale_s));
  }
  P.k_sum = a->k_sum;
  P.k_sum_scale = a->k_sum_scale;
  memcpy(P.k_sum_s, a->k_sum_stride, sizeof(P.k_sum_s));
  memcpy(P.k_sum_scale_s, a->k_sum_scale_stride, sizeof(P.k_sum_scale_s));
  P.chunk_tokens = a->chunk_tokens;
  P.tokens_before = a->tokens_before;
  P.row_base = a->row_base;
  P.page_table = a->page_table;
  P.status = a->status;
  P.n_chunks = a->n_chunks;
  P.n_layers = a->n_layers;
  P.n_heads = a->n_heads;
  P.n_tokens = a->n_tokens;
  P.head_dim = a->head_dim;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.pt_pages = row;
  P.n_pool_pages = a->n_pool_pages;
  P.n_units = (int32_t)units;
  P.pages = (int32_t)pages;
  P.fd_heads = kamera::make_fast_div((uint32_t)a->n_heads);
  P.fd_pages = kamera::make_fast_div((uint32_t)pages);
  P.fd_layers = kamera::make_fast_div((uint32_t)a->n_layers);
  launch = true;
  return KAMERA_OK;
}

// ---------------------------------------------------------------------------

// Sizes of a selection, and whether pages are scored apart.
int size_select(const kamera_select_args* a, bool& work, int32_t& n_pieces, int64_t& workspace) {
  const char* who = "kamera_select_pages";
  work = false;
  n_pieces = 0;
  workspace = 0;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_requests < 0 || a->n_keys < 0) return fail(KAMERA_ERR_SHAPE, "%s: negative n_requests/n_keys", who);
  int rc = check_head_dim(a->head_dim, who);
  if (rc) return rc;
  if ((rc = check_heads(a->n_q_heads, a->n_kv_heads, who))) return rc;
  if ((rc = check_page8(a->page_size, who))) return rc;
  if (a->n_first < 0 || a->n_last < 1 || (int64_t)a->n_first + a->n_last > a->n_keep)
    return fail(KAMERA_ERR_SHAPE, "%s: n_first %d >= 0 and n_last %d >= 1 pages must fit in n_keep %d", who, a->n_first,
                a->n_last, a->n_keep);
  const int64_t max_pages = ceil_div(a->n_keys, a->page_size);
  if (max_pages > KAMERA_MAX_SELECT_PAGES)
    return fail(KAMERA_ERR_RANGE, "%s: %lld pages a request exceed %d", who, (long long)max_pages,
                KAMERA_MAX_SELECT_PAGES);
  if (a->n_requests == 0) return KAMERA_OK;
  const int64_t wgs = bounded_product({a->n_requests, a->n_kv_heads});
  if (wgs < 0 || wgs * 1024 > 0xFFFFFFFFLL)
    return fail(KAMERA_ERR_RANGE, "%s: too many requests and heads for one launch", who);
  work = true;
  const int64_t pieces = ceil_div(max_pages, 256);
  if (max_pages > kSelectSplit && wgs <= 128 && max_pages > a->n_keep && wgs * pieces * 256 <= 0xFFFFFFFFLL) {
    n_pieces = (int32_t)pieces;
    workspace = wgs * max_pages * 4;
  }
  return KAMERA_OK;
}

int build_select(const kamera_select_args* a, kamera::SelectParams& P, bool& launch) {
  const char* who = "kamera_select_pages";
  bool work = false;
  int32_t n_pieces = 0;
  int64_t workspace = 0;
  launch = false;
  int rc = size_select(a, work, n_pieces, workspace);
  if (rc || !work) return rc;
  if ((rc = check_table(a->page_table, a->pt_stride, a->pt_stride, a->page_size, a->n_pool_pages, a->n_keys, who)))
    return rc;
  if (a->kv_tokens == nullptr || a->q == nullptr || a->k_sum == nullptr || a->k_sum_scale == nullptr ||
      a->sel == nullptr || a->sel_count == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: kv_tokens, q, k_sum, k_sum_scale, sel and sel_count are needed", who);
  if (!aligned16(a->k_sum) || !multiples(a->k_sum_stride, 2, 16))
    return fail(KAMERA_ERR_ALIGN, "%s: key sums must start at 16-byte boundaries", who);
  const int64_t wgs = (int64_t)a->n_requests * a->n_kv_heads;
  const int64_t entries = bounded_product({a->n_requests, a->n_kv_heads, a->n_keep});
  if (entries < 0) return fail(KAMERA_ERR_RANGE, "%s: n_keep too large", who);
  const int64_t ext_q[2] = {a->n_requests, a->n_q_heads}, ext_s[2] = {a->n_pool_pages, a->n_kv_heads};
  Range in[5] = {};
  if (!span(a->q, a->q_stride, ext_q, 2, a->head_dim, 2, in[0].lo, in[0].hi) ||
      !span(a->k_sum, a->k_sum_stride, ext_s, 2, a->head_dim, 1, in[1].lo, in[1].hi) ||
      !span(a->k_sum_scale, a->k_sum_scale_stride, ext_s, 2, 1, 4, in[2].lo, in[2].hi))
    return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  in[3] = table_range(a->page_table, a->n_requests, a->pt_stride, (int32_t)ceil_div(a->n_keys, a->page_size));
  in[4] = flat(a->kv_tokens, a->n_requests, 4);
  Range out[3] = {flat(a->sel, entries, 4), flat(a->sel_count, wgs, 4), {0, 0}};
  if (workspace > 0) {
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, workspace, who))) return rc;
    out[2] = flat(a->workspace, workspace, 1);
  }
  for (int i = 0; i < 3; ++i) {
    for (int k = 0; k < 5; ++k)
      if (meet(out[i], in[k])) return fail(KAMERA_ERR_ALIAS, "%s: an output or the workspace overlaps an input", who);
    for (int k = i + 1; k < 3; ++k)
      if (meet(out[i], out[k])) return fail(KAMERA_ERR_ALIAS, "%s: sel, sel_count and workspace overlap", who);
  }
  memset(&P, 0, sizeof(P));
  P.kv_tokens = a->kv_tokens;
  P.page_table = a->page_table;
  P.q = static_cast<const uint16_t*>(a->q);
  P.k_sum = a->k_sum;
  P.k_sum_scale = a->k_sum_scale;
  P.sel = a->sel;
  P.sel_count = a->sel_count;
  P.status = a->status;
  memcpy(P.q_s, a->q_stride, sizeof(P.q_s));
  memcpy(P.k_sum_s, a->k_sum_stride, sizeof(P.k_sum_s));
  memcpy(P.k_sum_scale_s, a->k_sum_scale_stride, sizeof(P.k_sum_scale_s));
  P.n_requests = a->n_requests;
  P.n_kv_heads = a->n_kv_heads;
  P.group = a->n_q_heads / a->n_kv_heads;
  P.head_dim = a->head_dim;
  P.n_keys = a->n_keys;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.n_pool_pages = a->n_pool_pages;
  P.n_keep = a->n_keep;
  P.n_first = a->n_first;
  P.n_last = a->n_last;
  P.max_pages = (int32_t)ceil_div(a->n_keys, a->page_size);
  P.n_pieces = n_pieces;
  P.keys = static_cast<uint32_t*>(a->workspace);
  launch = true;
  return KAMERA_OK;
}

// ---------------------------------------------------------------------------

// Sizes of an attention call, and how its work is split.
int size_attend(const kamera_attend_args* a, kamera::AttendParams& P, bool& launch, int64_t& workspace) {
  const char* who = "kamera_attend_paged";
  launch = false;
  workspace = 0;
  if (a == nullptr) return fail(KAMERA_ERR_NULL, "%s: args is NULL", who);
  if (a->n_requests < 0 || a->n_queries < 0 || a->n_keys < 0)
    return fail(KAMERA_ERR_SHAPE, "%s: negative n_requests/n_queries/n_keys", who);
  int rc = check_head_dim(a->head_dim, who);
  if (rc) return rc;
  if ((rc = check_heads(a->n_q_heads, a->n_kv_heads, who))) return rc;
  if (a->page_size <= 0 || a->page_size % 16 != 0)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: page_size must be a multiple of 16 (got %d)", who, a->page_size);
  if (a->cache_type != KAMERA_CACHE_BF16 && a->cache_type != KAMERA_CACHE_E4M3)
    return fail(KAMERA_ERR_SHAPE, "%s: unknown cache_type %d", who, a->cache_type);
  if (a->causal != 0 && a->causal != 1) return fail(KAMERA_ERR_SHAPE, "%s: causal must be 0 or 1", who);
  if (a->window < 0 || (a->window > 0 && !a->causal))
    return fail(KAMERA_ERR_SHAPE, "%s: a window must be positive and needs causal = 1", who);
  if (!isfinite(a->scale)) return fail(KAMERA_ERR_SHAPE, "%s: scale must be finite", who);
  if (a->n_splits < 0 || a->n_splits > 512) return fail(KAMERA_ERR_SHAPE, "%s: n_splits must be 0 .. 512", who);
  if (a->sel_stride < 0) return fail(KAMERA_ERR_SHAPE, "%s: negative sel_stride", who);
  if (a->sel_stride > 0 && a->n_queries > 1)
    return fail(KAMERA_ERR_UNSUPPORTED, "%s: selected pages serve one query token a request (n_queries %d)", who,
                a->n_queries);
  // token positions, and those of the part after the last one, stay in 31 bits
  if ((int64_t)a->n_keys + a->n_queries > INT32_MAX - 4096 ||
      (int64_t)a->sel_stride * a->page_size > INT32_MAX - 4096)
    return fail(KAMERA_ERR_RANGE, "%s: too many keys or queries a request", who);
  if (a->n_requests == 0 || a->n_queries == 0) return KAMERA_OK;
  const int group = a->n_q_heads / a->n_kv_heads;
  const int64_t rows = (int64_t)a->n_queries * group;
  if (rows > INT32_MAX / 2) return fail(KAMERA_ERR_RANGE, "%s: too many query rows", who);
  memset(&P, 0, sizeof(P));
  P.rows_max = (int32_t)rows;
  // Few rows or many.  The few-rows kernel takes 32 rows of an 8-bit cache at once
  // (4 queries of 8 heads, 32 requests of 8192 keys of 8 KV heads: 100 us, with the
  // other kernel 151; 5 queries: 158 and 153), and 16 of a bf16 one, whose loads leave
  // no registers for more (the same 4 queries: 209 us with the many-rows kernel, here 282
  // with two tiles a wave and 319 with one; 2 queries, 64 requests of 4096 keys: 193, here 201).
  const bool e4m3 = a->cache_type == KAMERA_CACHE_E4M3;
  P.tiles = rows > (e4m3 ? 32 : 16) && a->sel_stride == 0 ? 1 : 0;
  P.row_tiles = !P.tiles && e4m3 && rows > 16 ? 2 : 1;
  P.n_row_blocks = (int32_t)ceil_div(rows, P.tiles ? 128 : 16 * P.row_tiles);
  const int64_t tasks = bounded_product({a->n_requests, a->n_kv_heads, P.n_row_blocks});
  if (tasks < 0) return fail(KAMERA_ERR_RANGE, "%s: too many requests, heads and rows", who);
  if (a->n_splits > 0) {
    P.n_splits = a->n_splits;
  } else {
    // Few rows: one workgroup a CU, parts of at least 128 keys; up to 768 keys in 8
    // bits (384 in bf16) one part is as fast as many, which a second kernel joins (one
    // request of 8 KV heads, 8 bits, 1 / 8 / 16 / 32 parts: 512 keys 8.3 / 9.4 / 9.6 /
    // 9.7 us, 1024 keys 10.8 / 9.9 / 9.9 / 9.9, 4096 keys 27.4 / 12.2 / 11.1 / 10.4,
    // 16384 keys 96.5 / 21.6 / 16.4 / 13.7).  Many rows: two workgroups a CU, parts of
    // at least 512 keys.
    int64_t span_keys = a->sel_stride > 0 ? (int64_t)a->sel_stride * a->page_size : a->n_keys;
    if (a->window > 0) span_keys = std::min<int64_t>(span_keys, (int64_t)a->window + a->n_queries);
    const int64_t one = e4m3 ? 768 : 384;
    const int64_t most = P.tiles ? std::min<int64_t>(512 / tasks, span_keys / 512)
                                 : (span_keys <= one ? 1 : std::min<int64_t>(256 / tasks, span_keys / 128));
    P.n_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(most, 512));
  }
  int64_t wgs = bounded_product({tasks, P.n_splits});
  const int64_t join = bounded_product({a->n_requests, a->n_kv_heads, rows});
  if (P.tiles) {
    const int64_t pairs = (int64_t)a->n_requests * a->n_kv_heads;
    // every request's work on all XCDs alike, whatever the lengths
    P.deal = a->n_kv_heads % 8 == 0 ? 1 : (a->n_kv_heads % 4 == 0 ? 2 : (a->n_kv_heads % 2 == 0 ? 4 : 8));
    P.blocks_share = (int32_t)ceil_div(P.n_row_blocks, P.deal);
    wgs = bounded_product({pairs * P.deal, P.blocks_share, P.n_splits});
    P.n_shares = (int32_t)std::min<int64_t>(pairs * P.deal / 8, INT32_MAX);
  }
  // rows count only where a second kernel joins them
  if (wgs < 0 || wgs * 256 > 0xFFFFFFFFLL || (P.n_splits > 1 && (join < 0 || join * 256 > 0xFFFFFFFFLL)))
    return fail(KAMERA_ERR_RANGE, "%s: too many workgroups for one launch", who);
  P.n_tasks = (int32_t)wgs;
  P.n_join = P.n_splits > 1 ? (int32_t)join : 0;
  if (P.n_splits > 1) {
    workspace = bounded_product({join, P.n_splits, a->head_dim + 4, 4});
    if (workspace < 0) return fail(KAMERA_ERR_RANGE, "%s: workspace too large", who);
  }
  launch = true;
  return KAMERA_OK;
}

int build_attend(const kamera_attend_args* a, kamera::AttendParams& P, bool& launch) {
  const char* who = "kamera_attend_paged";
  int64_t workspace = 0;
  int rc = size_attend(a, P, launch, workspace);
  if (rc || !launch) return rc;
  launch = false;
  const bool e4m3 = a->cache_type == KAMERA_CACHE_E4M3;
  const int32_t row = row_pages(a->pt_stride, a->pt_pages);
  // selected pages are whatever sel holds: one past the row is not seen
  const int64_t tokens = a->sel_stride > 0 ? 0 : a->n_keys;
  if ((rc = check_table(a->page_table, a->pt_stride, row, a->page_size, a->n_pool_pages, tokens, who))) return rc;
  if (a->kv_tokens == nullptr || a->q == nullptr || a->out == nullptr || a->k_cache == nullptr || a->v_cache == nullptr)
    return fail(KAMERA_ERR_NULL, "%s: kv_tokens, q, out and the caches are needed", who);
  if (e4m3 && (a->k_scale == nullptr || a->v_scale == nullptr))
    return fail(KAMERA_ERR_NULL, "%s: an 8-bit cache needs its scales", who);
  if ((a->sel == nullptr) != (a->sel_count == nullptr) || (a->sel == nullptr) != (a->sel_stride == 0))
    return fail(KAMERA_ERR_NULL, "%s: sel, sel_count and sel_stride go together", who);
  if (!aligned16(a->q) || !aligned16(a->out) || !multiples(a->q_stride, 2, 8) || !multiples(a->out_stride, 2, 8))
    return fail(KAMERA_ERR_ALIGN, "%s: q and out rows must start at 16-byte boundaries", who);
  const int el = e4m3 ? 1 : 2;
  if (!aligned16(a->k_cache) || !aligned16(a->v_cache) || !multiples(a->k_cache_stride, 3, 16 / el) ||
      !multiples(a->v_cache_stride, 3, 16 / el))
    return fail(KAMERA_ERR_ALIGN, "%s: cache rows must start at 16-byte boundaries", who);
  // lane offsets within a 16-token part are 32-bit
  for (const int64_t t : {a->k_cache_stride[1], a->v_cache_stride[1]})
    if (t < 0 || t > (int64_t)1 << 24) return fail(KAMERA_ERR_RANGE, "%s: token stride %lld of the cache", who, (long long)t);
  const int64_t ext[3] = {a->n_pool_pages, a->page_size, a->n_kv_heads}, ext_s[2] = {a->n_pool_pages, a->n_kv_heads};
  // how far q, out and lse reach is known only without a row base
  const int64_t n_rows = a->q_base != nullptr ? a->n_queries : (int64_t)a->n_requests * a->n_queries;
  const int64_t ext_q[2] = {n_rows, a->n_q_heads};
  Range in[11] = {}, out[3] = {};
  if (!span(a->q, a->q_stride, ext_q, 2, a->head_dim, 2, in[0].lo, in[0].hi) ||
      !span(a->k_cache, a->k_cache_stride, ext, 3, a->head_dim, el, in[1].lo, in[1].hi) ||
      !span(a->v_cache, a->v_cache_stride, ext, 3, a->head_dim, el, in[2].lo, in[2].hi) ||
      !span(a->out, a->out_stride, ext_q, 2, a->head_dim, 2, out[0].lo, out[0].hi) ||
      (a->lse != nullptr && !span(a->lse, a->lse_stride, ext_q, 2, 1, 4, out[1].lo, out[1].hi)) ||
      (e4m3 && (!span(a->k_scale, a->k_scale_stride, ext_s, 2, 1, 4, in[3].lo, in[3].hi) ||
                !span(a->v_scale, a->v_scale_stride, ext_s, 2, 1, 4, in[4].lo, in[4].hi))))
    return fail(KAMERA_ERR_RANGE, "%s: strides span more than the address space", who);
  const int64_t entries = bounded_product({a->n_requests, a->n_kv_heads, a->sel_stride});
  if (entries < 0) return fail(KAMERA_ERR_RANGE, "%s: too many selected pages", who);
  in[5] = table_range(a->page_table, a->n_requests, a->pt_stride, row);
  in[6] = flat(a->kv_tokens, a->n_requests, 4);
  in[7] = flat_or(a->q_tokens, a->n_requests, 4);
  in[8] = flat_or(a->q_base, a->n_requests, 4);
  in[9] = flat_or(a->sel, entries, 4);
  in[10] = flat_or(a->sel_count, (int64_t)a->n_requests * a->n_kv_heads, 4);
  if (workspace > 0) {
    if ((rc = check_workspace(a->workspace, a->workspace_bytes, workspace, who))) return rc;
    out[2] = flat(a->workspace, workspace, 1);
  }
  for (int i = 0; i < 3; ++i) {
    for (const Range& r : in)
      if (meet(out[i], r)) return fail(KAMERA_ERR_ALIAS, "%s: out, lse or workspace overlaps an input", who);
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
  P.k = static_cast<const uint8_t*>(a->k_cache);
  P.v = static_cast<const uint8_t*>(a->v_cache);
  P.k_scale = a->k_scale;
  P.v_scale = a->v_scale;
  P.sel = a->sel;
  P.sel_count = a->sel_count;
  P.status = a->status;
  for (int k = 0; k < 2; ++k) {
    P.q_s[k] = a->q_stride[k];
    P.out_s[k] = a->out_stride[k];
    P.lse_s[k] = a->lse_stride[k];
    P.k_scale_s[k] = a->k_scale_stride[k];
    P.v_scale_s[k] = a->v_scale_stride[k];
  }
  for (int k = 0; k < 3; ++k) {
    P.k_s[k] = a->k_cache_stride[k] * el;
    P.v_s[k] = a->v_cache_stride[k] * el;
  }
  // the kernels take a largest score by its product with a positive factor; a
  // zero scale becomes one that leaves every score a difference of zero
  P.scale2 = std::max((float)(fabs((double)a->scale) * 1.4426950408889634074), 1e-30f);
  P.q_sign = a->scale < 0.f ? 0x80008000u : 0u;
  P.n_requests = a->n_requests;
  P.n_kv_heads = a->n_kv_heads;
  P.group = a->n_q_heads / a->n_kv_heads;
  P.head_dim = a->head_dim;
  P.n_queries = a->n_queries;
  P.n_keys = a->n_keys;
  P.page_size = a->page_size;
  P.pt_stride = a->pt_stride;
  P.pt_pages = row;
  P.n_pool_pages = a->n_pool_pages;
  P.cache_type = a->cache_type;
  P.causal = a->causal;
  P.window = std::min(a->window, std::max(a->n_keys, 1));   // a longer one sees no more, and positions less it could wrap
  P.sel_stride = a->sel_stride;
  if (workspace > 0) {
    const int64_t parts = (int64_t)a->n_requests * a->n_kv_heads * P.rows_max * P.n_splits;
    P.part_o = static_cast<float*>(a->workspace);
    P.part_ml = P.part_o + parts * a->head_dim;
  }
  P.fd_group = kamera::make_fast_div((uint32_t)P.group);
  P.fd_heads = kamera::make_fast_div((uint32_t)P.n_kv_heads);
  P.fd_blocks = kamera::make_fast_div((uint32_t)P.n_row_blocks);
  P.fd_splits = kamera::make_fast_div((uint32_t)P.n_splits);
  P.fd_rows = kamera::make_fast_div((uint32_t)P.rows_max);
  P.fd_shares = kamera::make_fast_div((uint32_t)std::max(P.n_shares, 1));
  P.fd_deal = kamera::make_fast_div((uint32_t)std::max(P.deal, 1));
  P.fd_page16 = kamera::make_fast_div((uint32_t)a->page_size / 16);
  launch = true;
  return KAMERA_OK;
}

int finish(hipError_t e, const char* who) {
  if (e != hipSuccess) return fail(KAMERA_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ok();
}

}  // namespace

extern "C" int kamera_page_tables(const kamera_page_tables_args* a, void* stream) {
  kamera::TablesParams P;
  bool launch = false;
  const int rc = build_tables(a, P, launch);
  if (rc) return rc;
  return finish(launch ? kamera::launch_page_tables(P, static_cast<hipStream_t>(stream)) : hipSuccess, "kamera_page_tables");
}

extern "C" int kamera_append_paged8(const kamera_append_args* a, void* stream) {
  kamera::AppendParams P;
  bool launch = false;
  const int rc = build_append(a, P, launch);
  if (rc) return rc;
  return finish(launch ? kamera::launch_append(P, static_cast<hipStream_t>(stream)) : hipSuccess, "kamera_append_paged8");
}

extern "C" int kamera_select_pages(const kamera_select_args* a, void* stream) {
  kamera::SelectParams P;
  bool launch = false;
  const int rc = build_select(a, P, launch);
  if (rc) return rc;
  return finish(launch ? kamera::launch_select(P, static_cast<hipStream_t>(stream)) : hipSuccess, "kamera_select_pages");
}

extern "C" int kamera_attend_paged(const kamera_attend_args* a, void* stream) {
  kamera::AttendParams P;
  bool launch = false;
  const int rc = build_attend(a, P, launch);
  if (rc) return rc;
  return finish(launch ? kamera::launch_attend(P, static_cast<hipStream_t>(stream)) : hipSuccess, "kamera_attend_paged");
}

extern "C" int64_t kamera_select_workspace(const kamera_select_args* a) {
  bool work = false;
  int32_t n_pieces = 0;
  int64_t workspace = 0;
  const int rc = size_select(a, work, n_pieces, workspace);
  if (rc) return rc;
  ok();
  return workspace;
}

extern "C" int64_t kamera_attend_workspace(const kamera_attend_args* a) {
  kamera::AttendParams P;
  bool launch = false;
  int64_t workspace = 0;
  const int rc = size_attend(a, P, launch, workspace);
  if (rc) return rc;
  ok();
  return workspace;
}

extern "C" int kamera_validate_cache(int32_t which, const void* args) {
  bool launch = false;
  int rc;
  switch (which) {
    case 0: { kamera::TablesParams P; rc = build_tables(static_cast<const kamera_page_tables_args*>(args), P, launch); break; }
    case 1: { kamera::AppendParams P; rc = build_append(static_cast<const kamera_append_args*>(args), P, launch); break; }
    case 2: { kamera::SelectParams P; rc = build_select(static_cast<const kamera_select_args*>(args), P, launch); break; }
    case 3: { kamera::AttendParams P; rc = build_attend(static_cast<const kamera_attend_args*>(args), P, launch); break; }
    default: return fail(KAMERA_ERR_SHAPE, "kamera_validate_cache: unknown entry point %d", which);
  }
  return rc ? rc : ok();
}
