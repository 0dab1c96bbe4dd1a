// Launch parameters of the kernels that serve from the paged cache (kernel
// arguments), built and validated by the host layer in kamera_cache.cpp.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "kamera_launch.h"

namespace kamera {

constexpr int kAppendThreads = 256;              // a workgroup of the append: a wave for each 16 tokens of a page
constexpr int append_units_wg(int page_size) { return kAppendThreads / 64 / (page_size / 16); }
constexpr int kMinExp = -100, kMaxExp = 120;     // exponents of the 8-bit cache's scales

struct TablesParams {
  const int32_t* tokens_before;
  const int32_t* tokens_after;
  const int32_t* free_pages;
  const int32_t* free_begin;
  int32_t* free_end;
  int32_t* page_table;
  int32_t* token_base;
  int64_t* slots;
  int64_t n_slots;
  uint32_t* status;
  int32_t n_requests, page_size, pt_stride, n_pool_pages, n_free;
  int32_t slots_aligned;             // to 16 bytes
  FastDiv fd_page;
};

struct AppendPlane {
  const uint16_t* rows;
  uint8_t* cache;
  float* scale;
  int64_t rows_s[4];
  int64_t cache_s[4];
  int64_t scale_s[3];
};

struct AppendParams {
  AppendPlane plane[2];              // keys, values
  int8_t* k_sum;                     // optional
  float* k_sum_scale;
  int64_t k_sum_s[3];
  int64_t k_sum_scale_s[3];
  const int32_t* chunk_tokens;
  const int32_t* tokens_before;
  const int32_t* row_base;
  const int32_t* page_table;
  uint32_t* status;
  int32_t n_chunks, n_layers, n_heads, n_tokens;
  int32_t head_dim, page_size, pt_stride, n_pool_pages;
  int32_t pt_pages;                  // entries of a table row
  int32_t n_units;                   // (chunk, layer, page of the chunk, plane, head): page_size / 16 waves each
  int32_t pages;                     // most pages that a chunk's new tokens touch
  FastDiv fd_heads, fd_pages, fd_layers;
};

struct SelectParams {
  const int32_t* kv_tokens;
  const int32_t* page_table;
  const uint16_t* q;
  const int8_t* k_sum;
  const float* k_sum_scale;
  int32_t* sel;
  int32_t* sel_count;
  uint32_t* status;
  int64_t q_s[2], k_sum_s[2], k_sum_scale_s[2];
  int32_t n_requests, n_kv_heads, group, head_dim;
  int32_t n_keys, page_size, pt_stride, n_pool_pages;
  int32_t n_keep, n_first, n_last;
  int32_t max_pages;                 // ceil(n_keys / page_size)
  int32_t n_pieces;                  // > 0: scored by workgroups of their own, so many a (request, KV head)
  uint32_t* keys;                    // [request][KV head][max_pages] of these
};

struct AttendParams {
  const int32_t* q_tokens;
  const int32_t* q_base;
  const int32_t* kv_tokens;
  const int32_t* page_table;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const uint8_t* k;
  const uint8_t* v;
  const float* k_scale;
  const float* v_scale;
  const int32_t* sel;
  const int32_t* sel_count;
  float* part_o;                     // [task row][split][D] unnormalised sums, n_splits > 1
  float* part_ml;                    // [task row][split][4] running maximum (in powers of 2), sum of the
                                     // rounded weights, sum of the weights
  uint32_t* status;
  int64_t q_s[2], out_s[2], lse_s[2];
  int64_t k_s[3], v_s[3];            // bytes: page, token, head
  int64_t k_scale_s[2], v_scale_s[2];
  float scale2;                      // |scale| * log2(e), at least 1e-30
  uint32_t q_sign;                   // 0x80008000 where the scale is negative: q's signs are turned
  int32_t n_requests, n_kv_heads, group, head_dim;
  int32_t n_queries, n_keys, page_size, pt_stride, n_pool_pages;
  int32_t pt_pages;                  // entries of a table row
  int32_t cache_type, causal, window, sel_stride;
  int32_t n_splits;
  int32_t rows_max;                  // n_queries * group: rows of one (request, KV head)
  int32_t tiles;                     // 1: the many-rows kernel
  int32_t row_tiles;                 // few-rows kernel: tiles of 16 rows a wave, 1 or 2
  int32_t n_row_blocks;
  int32_t n_tasks;                   // workgroups
  int32_t n_join;                    // rows of all requests and KV heads (n_splits > 1)
  int32_t deal;                      // many-rows kernel: shares that a (request, KV head) pair's row blocks
  int32_t n_shares;                  // are dealt into, shares on an XCD, row blocks of a share
  int32_t blocks_share;
  FastDiv fd_group, fd_heads, fd_blocks, fd_splits, fd_rows, fd_shares, fd_deal;
  FastDiv fd_page16;                 // by page_size / 16
};

hipError_t launch_page_tables(const TablesParams& p, hipStream_t s);
hipError_t launch_append(const AppendParams& p, hipStream_t s);
hipError_t launch_select(const SelectParams& p, hipStream_t s);
hipError_t launch_attend(const AttendParams& p, hipStream_t s);
hipError_t launch_attend_tiles(const AttendParams& p, hipStream_t s);   // by launch_attend

}  // namespace kamera
