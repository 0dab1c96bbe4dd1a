// Launch parameters of the kernels that serve from a paged latent cache (kernel
// arguments), built and validated by the host layer in kamera_latent.cpp.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "kamera_launch.h"

namespace kamera {

constexpr int kRopeCols = 64;        // columns of the rope key behind a latent

// ---- rotated append ----

constexpr int kRotateTokens = 32;    // most tokens of a workgroup

struct RotatePlane {
  const uint16_t* in;
  uint16_t* out;
  int64_t in_s[4];                   // chunk, layer, row, head
  int64_t out_s[4];                  // the same (queries); layer, page, token, head (pool)
  int32_t n_heads;                   // 0: the plane is not there
  int32_t n_items;                   // threads' pieces of a head's row: the band's first, then 16-byte copies
  int32_t band_items;
  int32_t band_vec;                  // first 16-byte vector of the band
  FastDiv fd_heads, fd_items;
};

struct RotateParams {
  RopeParams rope;
  RotatePlane plane[3];              // keys, values, queries
  const int32_t* chunk_tokens;
  const int32_t* tokens_before;
  const int32_t* row_base;
  const int32_t* page_table;
  const int32_t* positions;
  int64_t position_s[3];
  uint32_t* status;
  float amplitude;
  int32_t n_tokens, page_size, pt_stride, pt_pages, n_pool_pages;
  int32_t n_layers, n_blocks;
  int32_t block_tokens;              // tokens of a workgroup
  int32_t n_tasks;
  FastDiv fd_blocks, fd_layers, fd_page;
};

// ---- products ----

struct ProjectParams {
  const uint16_t* x;
  const uint16_t* w;
  uint16_t* out;
  int64_t x_s[2];                    // row, head (dense); page, token (paged)
  int64_t w_s[3];
  int64_t out_s[2];
  // paged
  const int32_t* kv_tokens;
  const int32_t* row_base;
  const int32_t* page_table;
  uint32_t* status;
  int32_t n_requests, n_keys, page_size, pt_stride, n_pool_pages;
  int32_t n_rows, n_heads, n_in, n_out;
  int32_t paged;
  int32_t w_k;                       // 1: W's columns of one output lie together (stride `in` is 1)
  int32_t tile_rows;                 // 32, 128 (tiles of 128 columns) or 256 (of 256)
  int32_t n_row_blocks, n_col_blocks;
  int32_t n_tasks, per_xcd;
  FastDiv fd_rows, fd_cols, fd_heads, fd_page;
};

// ---- attention ----

// From so many (request, head, row block) tasks on a workgroup takes one whole.  Whole tasks keep the row blocks of a
// head, which read the same keys, together in time; divided ones end together.  Which counts for more depends on lengths
// that the host does not know (us whole / divided).  Expanded: prompts of 1024 queries over 4096 keys, 2048 equal tasks
// 622 / 738, 1024 tasks 319 / 353; ragged prompts, 1024 tasks 146 / 122, 2048 tasks 238 / 197, 4096 of 16 requests 602 /
// 467; 128 heads, two prompts of 1024 (2048 tasks) 150 / 139, four ragged ones (6656) 486 / 247.  Latent: 2048 single
// queries of 16 heads over 1024 keys 441 / 488, over 1 to 2047 484 / 496, over 1 to 8191 1647 / 1629; of 128 heads over
// 2048 keys 1412 / 1425, over 1 to 4095 1673 / 1499; 64 prompts of 64 queries of 128 heads (4096 tasks) 1275 / 1392,
// ragged 1303 / 1448.
constexpr int kMlaDivideTasks = 2048;

// Latent form: waves of a workgroup whose row blocks are `row_waves` waves (of 16 rows) high,
// and its groups, which take 32 keys in turn.
constexpr int latent_waves(int row_waves) { return row_waves == 8 ? 8 : 4; }
constexpr int latent_groups(int row_waves) { return latent_waves(row_waves) / row_waves; }

struct MlaParams {
  const int32_t* q_tokens;
  const int32_t* q_base;
  const int32_t* kv_tokens;
  const int32_t* kv_base;            // expanded
  const int32_t* page_table;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const uint8_t* pool;               // latent rows, or the rope columns (expanded)
  const uint8_t* k;                  // expanded
  const uint8_t* v;
  float* part_o;                     // [workgroup][2][rows of a block][columns] unnormalised sums
  float* part_ml;                    // [workgroup][2][rows of a block][4] running maximum (in powers of 2), sum of
                                     // the rounded weights, sum of the weights
  int32_t* prefix;                   // [n_tasks] cost before each task, cost of a workgroup, [n_parts] first tasks
  uint32_t* status;
  int64_t q_s[2], out_s[2], lse_s[2];
  int64_t pool_s[2];                 // bytes: page, token
  int64_t k_s[2], v_s[2];            // bytes: row, head
  float scale2;                      // |scale| * log2(e), at least 1e-30
  uint32_t q_sign;                   // 0x80008000 where the scale is negative: q's signs are turned
  int32_t n_requests, n_heads, dim;  // dim: latent_dim or head_dim
  int32_t n_queries, n_keys, page_size, pt_stride, n_pool_pages;
  int32_t causal, window;
  int32_t group;                     // heads of a token that are rows of one task (latent: all, expanded: 1)
  int32_t task_heads;                // heads that are tasks of their own (latent: 1, expanded: all)
  int32_t rows_block;                // rows of a task
  int32_t row_waves;                 // latent: waves of a row block, 1, 2 or 8
  int32_t n_row_blocks;
  int32_t n_tasks;
  int32_t n_parts;                   // > 0: workgroups among which all tasks' cost is divided; 0: one a task
  int32_t min_units;                 // least cost of a workgroup
  int32_t unit;                      // keys of a unit
  int32_t fixed;                     // units that a task costs beside its own
  int32_t lanes;                     // of a wave that add up a request's units: a power of two up to 64
  FastDiv fd_group, fd_blocks, fd_heads, fd_page16;
};

hipError_t launch_rotate(const RotateParams& p, hipStream_t s);
hipError_t launch_project(const ProjectParams& p, hipStream_t s);
hipError_t launch_attend_latent(const MlaParams& p, hipStream_t s);
hipError_t launch_attend_expanded(const MlaParams& p, hipStream_t s);
hipError_t launch_mla_join(const MlaParams& p, hipStream_t s);      // by the two above

}  // namespace kamera
