/*
 * kamera.h -- C ABI of the Kamera chunk-reuse operator for AMD Instinct MI355X
 * (gfx950).
 *
 * Kamera (arxiv 2606.23581) stores each cached chunk position-free -- the
 * pre-RoPE keys and the values of every layer and KV head, or an MLA latent
 * plus its decoupled rope key -- together with a rank-m "conditioning patch"
 * per layer and head (Eq. eq:operator, Sec. 1; Sec. 3).  Reusing the chunk at
 * a new position needs no forward pass: the keys are re-rotated to the target
 * position and the patch is added back (App. A, serve step).  This library
 * performs that serve step on the GPU:
 *
 *   kamera_rehydrate     K' = R(pos) (K + U_k W_k),  V' = V + U_v W_v,
 *                        into a dense buffer or straight into a paged KV pool;
 *                        with a per-chunk delta it relocates already-rotated
 *                        keys and adds a (removal) patch (Sec. 5, Table evict);
 *   kamera_shift         K' = R(delta) K, in place, for keys that are already
 *                        rotated (R(delta) R(p) = R(p + delta), Sec. 1 and 3:
 *                        reorder, sliding-window survivors, Sec. 5);
 *   kamera_scatter_paged a bit copy of dense token rows into the pool slots a
 *                        page table names (the clean-view overwrite, App. E),
 *   kamera_gather_paged  and the copy back from the pool into dense rows;
 *   kamera_form_patch    the compile step's truncated SVD of given deficits
 *                        (App. A), also as one orbit patch over orderings
 *                        (Sec. 5, reorder).
 *
 * and, for the program that goes on to answer from the cache:
 *
 *   kamera_page_tables   pages and token slots for requests that grow;
 *   kamera_append_paged8 bf16 K, V rows into a paged cache held in 8 bits;
 *   kamera_select_pages  the pages a query needs most, by a cheap score;
 *   kamera_attend_paged  attention over the paged cache (8 bits or bf16).
 *
 * Conventions shared by every entry point
 *   - Every tensor pointer is a DEVICE pointer owned by the caller.  The
 *     library never allocates, frees or synchronises; a call enqueues its
 *     kernel (kamera_form_patch: two or three, one after the other;
 *     kamera_select_pages and kamera_attend_paged: two where split) on
 *     `stream` (a hipStream_t; NULL = the default stream) and returns.  Results are
 *     visible to later work on that stream.
 *   - KV rows are bf16.  Strides are in ELEMENTS (bf16) unless named _bytes;
 *     the innermost (column) stride is always 1.  Row starts must be 16-byte
 *     aligned: base pointers 16-byte aligned and every stride a multiple of 8.
 *   - Per-chunk integers (positions, deltas, row bases, token counts, page
 *     tables) are int32 arrays in device memory.
 *   - Return value: KAMERA_OK (0) or a negative kamera_status.  Argument
 *     errors are detected on the host BEFORE any HIP call, so a failed call
 *     has no side effect; kamera_last_error() then describes the problem.
 *   - Calls are thread-safe; the error text is per thread.
 *   - Contents of device arrays (page-table entries, positions) cannot be
 *     checked on the host.  Page numbers outside [0, n_pool_pages) are
 *     skipped by the kernels and flagged in the optional `status` word
 *     (bit KAMERA_STATUS_BAD_PAGE), never written out of bounds.  A page
 *     table must be injective for the result to be defined;
 *     kamera_check_page_table() verifies a host copy.
 */
#ifndef KAMERA_H
#define KAMERA_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KAMERA_ABI_VERSION 4

/* Largest patch rank m accepted (>= the 128-wide head, so a full-rank patch
 * that reproduces any Delta K exactly can be applied). */
#define KAMERA_MAX_RANK 128
/* Rotated band width limit and row width limit, in elements. */
#define KAMERA_MAX_ROPE_DIM 128
#define KAMERA_MAX_HEAD_DIM 4096

typedef enum {
  KAMERA_OK = 0,
  KAMERA_ERR_NULL = -1,        /* a required pointer is NULL                    */
  KAMERA_ERR_SHAPE = -2,       /* inconsistent sizes, bands or sections         */
  KAMERA_ERR_ALIGN = -3,       /* pointer or stride breaks 16-byte row alignment */
  KAMERA_ERR_RANGE = -4,       /* a size or rank beyond the supported maximum    */
  KAMERA_ERR_ALIAS = -5,       /* an output overlaps an input it must not        */
  KAMERA_ERR_UNSUPPORTED = -6, /* a valid request this library does not implement */
  KAMERA_ERR_HIP = -7          /* the HIP runtime refused the launch             */
} kamera_status;

/* bits of the optional device status word */
#define KAMERA_STATUS_BAD_PAGE 1u

typedef enum {
  KAMERA_PAIR_NEOX = 0,        /* pair j = columns (j, j + rope_dim/2)          */
  KAMERA_PAIR_INTERLEAVED = 1  /* pair j = columns (2j, 2j + 1)                 */
} kamera_pairing;

typedef enum {
  KAMERA_SECTIONS_BLOCKED = 0,     /* pairs [0,s0) use t, [s0,s0+s1) h, rest w  */
  KAMERA_SECTIONS_INTERLEAVED = 1  /* pairs cycle t,h,w, skipping a coordinate
                                      whose section count is used up            */
} kamera_section_order;

typedef enum {
  KAMERA_POS_LINEAR = 0,   /* token i at p0 + i on every coordinate;
                              chunk_pos[c*3 + 0] = p0                         */
  KAMERA_POS_GRID3 = 1,    /* token i at (t0, h0 + i / grid_w, w0 + i % grid_w);
                              chunk_pos[c*3 + 0..2] = (t0, h0, w0)            */
  KAMERA_POS_EXPLICIT = 2  /* token i of chunk c at explicit_pos[c*explicit_
                              chunk_stride + i*3 + (0,1,2)]                   */
} kamera_pos_mode;

/* Which rehydrate kernel a call uses.  Both compute the same bits.
 * PER_HEAD: one workgroup per (plane, chunk, layer, head, token block, column
 * block); any row layout.  ROW_GROUP: one workgroup per (plane, chunk, layer,
 * token block) taking every head of a token row, so that a 16-token pool page
 * is written as one contiguous run; possible for rows of <= 8 heads of 128
 * columns (one block per head, the rope band if any being the whole head),
 * rank <= 64 in whole 16-byte U chunks, linear or grid positions (with or
 * without relocation), and byte offsets below 2^31 within one (chunk, layer)
 * slab or one layer of the pool.  A row-group workgroup takes 8 heads (one per CU),
 * or 4 (two per CU; rows of <= 4 heads, or 8 heads in two groups).  AUTO
 * takes ROW_GROUP4 where it was measured faster on MI355X: rows of 4 or 8
 * heads, chunks of >= 256 tokens and >= 2^19 rows in all (planes x chunks x
 * layers x tokens x heads), except dense outputs at rank <= 32 with 2^21 to
 * 2^23 rows.  Those, fewer rows, shorter chunks and other head counts keep
 * PER_HEAD.  A ROW_GROUP or ROW_GROUP4 request that is not possible falls
 * back to PER_HEAD. */
typedef enum {
  KAMERA_KERNEL_AUTO = 0,
  KAMERA_KERNEL_PER_HEAD = 1,
  KAMERA_KERNEL_ROW_GROUP = 2,   /* 8 heads per workgroup (4 for rows of <= 4) */
  KAMERA_KERNEL_ROW_GROUP4 = 3   /* 4 heads per workgroup, also for wider rows */
} kamera_kernel_choice;

/* How the row-group kernel spreads its work over the device (same bits
 * either way).  PERSISTENT: one resident wave of workgroups, each walking an
 * equal share (in bytes moved) of its (plane, head group)'s 16-token tiles,
 * so that a unit's set-up (W^T, page numbers) is paid once per long range
 * and every workgroup finishes together.  BLOCKS: one workgroup per token
 * block of one (plane, chunk, layer, head group), blocks of up to 1024 tokens
 * shrunk (to >= 64) until the launch has 4096 of them (2048 with 8-head
 * groups), handed out by the hardware as workgroups finish.  AUTO takes
 * BLOCKS where those blocks stay >= 512 tokens (long launches, where it
 * measured faster) and PERSISTENT otherwise, or whenever max_workgroups > 0.
 * The per-head kernel ignores the field. */
typedef enum {
  KAMERA_SCHEDULE_AUTO = 0,
  KAMERA_SCHEDULE_PERSISTENT = 1,
  KAMERA_SCHEDULE_BLOCKS = 2
} kamera_row_schedule;

typedef enum {
  KAMERA_PATCH_PRE_ROPE = 0,  /* K' = R(pos)(K + U W): the patch lives in the
                                 stored, position-free frame (Sec. 3)         */
  KAMERA_PATCH_POST_ROPE = 1  /* K' = R(pos) K + U W: the literal form of
                                 Eq. eq:operator, and the frame of a key
                                 deficit taken against R(pos) K as App. A's
                                 compile step does (see kamera_form_patch)    */
} kamera_patch_frame;

/* RoPE variant (Sec. 3 content | RoPE split; Fig. fig:unify for M-RoPE).
 * Pair j has frequency theta^(-2j/rope_dim) and rotates by angle
 * coord(j) * frequency, x' = x cos - y sin, y' = x sin + y cos. */
typedef struct {
  double theta;            /* rotary base, > 1                                */
  int32_t rope_offset;     /* first rotated column (0 for GQA/MHA, 512 MLA)  */
  int32_t rope_dim;        /* rotated width: even, <= KAMERA_MAX_ROPE_DIM    */
  int32_t pairing;         /* kamera_pairing                                 */
  int32_t n_sections;      /* 1: 1-D RoPE (coordinate t); 3: (t, h, w)       */
  int32_t sections[3];     /* pair counts of t, h, w; sum = rope_dim / 2     */
  int32_t section_order;   /* kamera_section_order                           */
} kamera_rope;

/* One stream of rows the call rebuilds: the keys (rotate = 1) or the values
 * (rotate = 0).  Element (c, l, i, h, col) of the input sits at
 *   in + c*in_stride[0] + l*in_stride[1] + i*in_stride[2] + h*in_stride[3] + col.
 * The patch factors of (c, l, h): U is n x m (token i, rank k) at
 *   U + c*u_stride[0] + l*u_stride[1] + h*u_stride[2] + i*u_stride[3] + k,
 * W is m x patch_dim at
 *   W + c*w_stride[0] + l*w_stride[1] + h*w_stride[2] + k*w_stride[3] + col',
 * col' = col - patch_offset.  A stride of 0 shares a factor (e.g. one basis
 * per layer for every chunk).  m = 0 disables the patch (U, W may be NULL).
 *
 * A plane covers the columns [col_begin, col_end) of the row (both 0: the
 * whole row; otherwise multiples of 32).  Two planes over the same rows with
 * disjoint column ranges give one row two patches of different rank, e.g. the
 * MLA latent (rank m) and the small extra patch on its rope key band that
 * Sec. 3 adds to close the latent-only residual.
 *
 * layer_rank (optional device int32 [n_layers]) lowers the rank per layer:
 * layer l uses the first min(layer_rank[l], m) ranks, 0 = no patch at that
 * layer -- the deep-half patch that stores factors for the deepest layers
 * only (Sec. 1 contributions, Table menu). */
typedef struct {
  const void* in;
  int64_t in_stride[4];
  void* out;               /* dense or pool base, see kamera_rehydrate_args  */
  int64_t out_stride[4];
  const void* U;
  int64_t u_stride[4];
  const void* W;
  int64_t w_stride[4];
  int32_t m;               /* patch rank, 0 .. KAMERA_MAX_RANK               */
  int32_t rotate;          /* 1: rotate the rope band (keys); 0: values      */
  int32_t patch_offset;    /* patched columns [patch_offset,                 */
  int32_t patch_dim;       /*                  patch_offset + patch_dim)     */
  int32_t col_begin;       /* columns this plane covers (0, 0: all)          */
  int32_t col_end;
  const int32_t* layer_rank;
} kamera_plane;

/* kamera_rehydrate -- Eq. eq:operator with the patch in the stored frame;
 * the serve step of App. A for every (chunk, layer, KV head) at once.
 *
 * Output destination of token i of chunk c, layer l, head h:
 *   dense (paged = 0): out + c*out_stride[0] + l*out_stride[1]
 *                          + (row_base[c] + i)*out_stride[2] + h*out_stride[3]
 *                      (row_base NULL = 0 for every chunk)
 *   paged (paged = 1): slot = page_table[c*pt_stride + i/page_size]*page_size
 *                             + i % page_size,
 *                      out + l*out_stride[1] + slot*out_stride[2]
 *                          + h*out_stride[3]   (out_stride[0] unused)
 * Outputs must not overlap inputs (checked on the extents the host-visible
 * sizes imply), except exactly in place: a dense output with row_base NULL,
 * the same base pointer and the same strides as the input (each element is
 * then read and written by the same workgroup; two planes in place on one
 * tensor must cover disjoint columns).  The two planes' outputs must not
 * overlap each other either, except (a) one tensor through the same mapping
 * on disjoint columns, or (b) interleaved rows: the same out_stride, all of
 * them >= 0, the layer (and for dense output the chunk) stride a multiple of
 * the row stride out_stride[2], and the bases d elements apart with
 * span <= |d| and |d| + span <= out_stride[2], span = (n_heads - 1) *
 * out_stride[3] + head_dim -- e.g. a pool [layer][slot][K|V][head][dim] in
 * which the K and V rows of a slot are adjacent, so that a page of both
 * planes is one contiguous run.  By the same rule a dense output may
 * interleave with the other plane's input (one tensor [chunk][layer][token]
 * [K|V][head][dim] rehydrated in place, each plane exactly in place).
 *
 * Relocation (delta != NULL, device int32 [n_chunks][3]): the input keys are
 * already rotated, at target - delta (survivors of a window slide, Sec. 5),
 * and the rotated planes compute
 *   K' = R(delta) K + R(target) U W      (KAMERA_PATCH_PRE_ROPE), or
 *   K' = R(delta) K + U W                (KAMERA_PATCH_POST_ROPE),
 * i.e. the move of kamera_shift fused with a (removal) patch (Sec. 5, Table
 * evict); target positions come from pos_mode as usual.  Unrotated planes
 * (values, latents) are unaffected by delta. */
typedef struct {
  int32_t n_chunks;
  int32_t n_layers;
  int32_t n_heads;             /* KV heads (1 for an MLA latent row)          */
  int32_t head_dim;            /* row width in elements, multiple of 32       */
  int32_t n_tokens;            /* tokens per chunk (the maximum if ragged)     */
  const int32_t* chunk_tokens; /* device [n_chunks] (<= n_tokens) or NULL      */
  int32_t patch_frame;         /* kamera_patch_frame                           */
  kamera_rope rope;
  int32_t pos_mode;            /* kamera_pos_mode                              */
  const int32_t* chunk_pos;    /* device [n_chunks][3] (LINEAR, GRID3)         */
  int32_t grid_w;              /* GRID3 tokens per grid row, > 0               */
  const int32_t* explicit_pos; /* device (EXPLICIT)                            */
  int64_t explicit_chunk_stride;
  int32_t n_planes;            /* 1 (keys only, e.g. MLA) or 2 (keys, values)  */
  kamera_plane plane[2];
  int32_t paged;
  const int32_t* row_base;     /* dense: device [n_chunks] or NULL             */
  const int32_t* page_table;   /* paged: device [n_chunks][pt_stride]          */
  int32_t pt_stride;
  int32_t page_size;
  int32_t n_pool_pages;
  uint32_t* status;            /* optional device word, bits OR-ed in          */
  const int32_t* delta;        /* optional: relocation of rotated keys         */
  int32_t kernel;              /* kamera_kernel_choice (0: AUTO)               */
  int32_t max_workgroups;      /* row-group kernel, persistent schedule: 0 =
                                  one resident wave of workgroups on the whole
                                  device, > 0 = at most this many (leaves CUs
                                  to concurrent work); same results.  Not
                                  allowed with KAMERA_SCHEDULE_BLOCKS
                                  (KAMERA_ERR_SHAPE).  The per-head kernel
                                  launches one workgroup per task and ignores
                                  it.                                         */
  int32_t schedule;            /* kamera_row_schedule (0: AUTO)                */
} kamera_rehydrate_args;

/* kamera_shift -- K' = R(delta_c) K in place on the rope band of every token
 * of every listed chunk (Sec. 1, Sec. 3; survivors of a window slide, Sec. 5).
 * Columns outside the band and the values are never touched.
 * delta: device [n_chunks][3] int32, the move of (t, h, w); 1-D RoPE reads
 * delta[c*3 + 0].  Token i of chunk c is row
 *   dense: k + c*k_stride[0] + l*k_stride[1] + (row_base[c] + i)*k_stride[2]
 *            + h*k_stride[3]          (row_base NULL = 0)
 *   paged: k + l*k_stride[1] + slot*k_stride[2] + h*k_stride[3],
 *          slot as in kamera_rehydrate. */
typedef struct {
  int32_t n_chunks;
  int32_t n_layers;
  int32_t n_heads;
  int32_t head_dim;
  int32_t n_tokens;
  const int32_t* chunk_tokens;
  kamera_rope rope;
  const int32_t* delta;
  void* k;
  int64_t k_stride[4];
  int32_t paged;
  const int32_t* row_base;
  const int32_t* page_table;
  int32_t pt_stride;
  int32_t page_size;
  int32_t n_pool_pages;
  uint32_t* status;
} kamera_shift_args;

/* kamera_scatter_paged / kamera_gather_paged -- bit-exact copies between
 * dense token rows and a paged pool (the copy half of the conditioning
 * switch, App. E: the clean view is restored by a plain copy; the pool is the
 * paged KV store the serve step writes into, Sec. 6).  For token i of chunk
 * c, layer l the dense row is
 *   rows + c*rows_stride_bytes[0] + l*rows_stride_bytes[1] + i*rows_stride_bytes[2]
 * and the pool row pool + l*pool_stride_bytes[0] + slot*pool_stride_bytes[1],
 * slot as in kamera_rehydrate; row_bytes bytes move, dense -> pool (scatter)
 * or pool -> dense (gather).  row_bytes and all strides: multiples of 16. */
typedef struct {
  int32_t n_chunks;
  int32_t n_layers;
  int32_t n_tokens;
  const int32_t* chunk_tokens;
  int64_t row_bytes;
  void* rows;
  int64_t rows_stride_bytes[3];
  void* pool;
  int64_t pool_stride_bytes[2];
  const int32_t* page_table;
  int32_t pt_stride;
  int32_t page_size;
  int32_t n_pool_pages;
  uint32_t* status;
} kamera_scatter_args;

/* kamera_form_patch -- the compile step of App. A on given deficits: for
 * every (chunk, layer, head) unit, the top-m singular triplets of
 * Delta (n x dim, fp32) as the stored patch
 *   U = U_svd[:, :m] * S[:m]   (n x m, bf16, singular values folded in),
 *   W = Vt[:m]                 (m x dim, bf16),
 * so U W is the best rank-m approximation of Delta.  The conditioned forward
 * pass that produces Delta needs model weights and is not part of this
 * library.
 * Frame of the factors: U W lives in the frame Delta was taken in, and the
 * kamera_rehydrate call that applies it must use the same frame.
 *   - App. A takes the key deficit against the canonical keys already turned
 *     to the target, Delta = K_cond - R(p) K: the rotated frame.  Such
 *     factors are applied with KAMERA_PATCH_POST_ROPE, K' = R(p) K + U W, at
 *     the positions p they were formed at.
 *   - For the default KAMERA_PATCH_PRE_ROPE, K' = R(p)(K + U W), turn each
 *     token's deficit back first, Delta_i <- R(-p_i) Delta_i (row i at its
 *     position p_i); the patch formed from that serves every position.
 *   Applying rotated-frame factors with KAMERA_PATCH_PRE_ROPE rotates the
 *   patch a second time and gives wrong keys.  Values and the MLA latent are
 *   never rotated, so for them the two frames coincide.
 * Layouts: element (c, l, h, i, j) of Delta at delta + c*delta_stride[0] +
 * l*delta_stride[1] + h*delta_stride[2] + i*delta_stride[3] + j (fp32,
 * 16-byte aligned rows); U and W as in kamera_plane (bf16); sigma (optional,
 * fp32) receives S[:m] at sigma + c*sigma_stride[0] + l*sigma_stride[1] +
 * h*sigma_stride[2] + k.  Method: the Gram matrix Delta^T Delta in fp32,
 * then its m largest eigenpairs, by one of two fp32 solvers:
 *   sweeps = 0 (default): Householder reduction to tridiagonal form,
 *     multisection on Sturm counts for the eigenvalues, twisted
 *     factorisation for their eigenvectors (close eigenvalues, within 1e-3 of
 *     the spectral norm, reorthogonalised), back-transformation; a unit whose vectors fail its
 *     checks (exactly multiple eigenvalues) is formed again by block Jacobi
 *     in a launch of its own;
 *   sweeps > 0: block cyclic Jacobi, at most `sweeps` sweeps, stopping once
 *     the off-diagonal mass is negligible (12 reach the fp32 floor here).
 * Either way singular vectors are accurate to ~1e-5 relative where the
 * spectrum has a gap at m.  W = V_m^T (bf16) is written first; U = Delta W^T
 * is then formed from that stored W in a later launch on the same stream
 * (Delta enters as a two-part bf16 split, ~2^-16 relative), so that U W is
 * the projection onto exactly the kept W.
 * Orbit patch (Sec. 5, reorder): with n_orbit = K >= 2 the deficits of K
 * orderings of the same chunk set, at delta + o*orbit_stride (o < K), are
 * averaged (fp32) and the mean is truncated as above: the one rank-m patch
 * with the least total squared error over those orderings.  A held-out
 * ordering is simply not passed.  n_orbit 0 or 1 = a single deficit.
 * U, W and sigma must not overlap the deficits, nor U overlap W
 * (KAMERA_ERR_ALIAS). */
#define KAMERA_FORM_MAX_DIM 128
typedef struct {
  int32_t n_chunks;
  int32_t n_layers;
  int32_t n_heads;
  int32_t n_tokens;            /* rows n of each Delta                          */
  int32_t dim;                 /* columns: multiple of 4, <= KAMERA_FORM_MAX_DIM */
  int32_t m;                   /* rank kept: 1 .. dim                           */
  int32_t sweeps;              /* 0 = tridiagonal solver, > 0 = Jacobi limit   */
  int32_t n_orbit;             /* deficits averaged per unit (0 or 1 = one)     */
  const float* delta;
  int64_t delta_stride[4];
  void* U;
  int64_t u_stride[4];
  void* W;
  int64_t w_stride[4];
  float* sigma;
  int64_t sigma_stride[3];
  int64_t orbit_stride;        /* elements between orbit members of delta       */
  int32_t* sweeps_done;        /* optional: Jacobi sweeps each unit ran (0 with
                                  the tridiagonal solver), dense
                                  [n_chunks][n_layers][n_heads] int32          */
} kamera_form_args;

int kamera_rehydrate(const kamera_rehydrate_args* args, void* stream);
int kamera_form_patch(const kamera_form_args* args, void* stream);
int kamera_shift(const kamera_shift_args* args, void* stream);
int kamera_scatter_paged(const kamera_scatter_args* args, void* stream);
int kamera_gather_paged(const kamera_scatter_args* args, void* stream);

/* ------------------------------------------------------------------------
 * Serving from the paged cache: pages for requests, the cache in 8 bits, and
 * attention over it.
 *
 * The 8-bit cache.  A page holds page_size (16, 32 or 64) tokens of one layer
 * as e4m3 bytes (4 exponent and 3 fraction bits, largest value 448, no
 * infinity; NaN is 0x7f / 0xff), with ONE fp32 scale for each (page, KV head)
 * and plane: value = byte * scale.  Scales are powers of two, 2^e with
 * -100 <= e <= 120, and e is the least exponent at which the page's largest
 * finite magnitude is at most 448 * 2^e.  A byte's value, its scaling to bf16
 * and a later change of e by whole steps are therefore exact wherever the
 * byte stays a normal number, and none of it depends on an order of summation:
 * the stored bytes are a function of the rows and of how they were divided over
 * calls.  (A call whose rows raise a page's e rounds the bytes there a second
 * time, where they leave the normal range; rows that come in one call, or
 * without a larger magnitude after them, are rounded once.)
 * Element (layer l, page p, token t of the page, head h, column j) is at
 *   base + l*stride[0] + p*stride[1] + t*stride[2] + h*stride[3] + j,
 * any strides that are multiples of 16 bytes (e.g. [layer][page][head][token]
 * [dim], which keeps what one (page, head) needs together, or the row order
 * [layer][slot][head][dim] of the bf16 pool).
 * ------------------------------------------------------------------------ */

/* further bits of the optional device status word */
#define KAMERA_STATUS_NO_PAGE 2u     /* the free list ran out                  */
#define KAMERA_STATUS_BAD_LENGTH 4u  /* a request outgrew its page-table row   */

/* Most requests of one kamera_page_tables call. */
#define KAMERA_MAX_REQUESTS 8192
/* Most pages of one request in kamera_select_pages (scores are kept in LDS). */
#define KAMERA_MAX_SELECT_PAGES 32768
/* Most query heads that share a KV head. */
#define KAMERA_MAX_GROUP 64

/* kamera_page_tables -- pages and token slots for requests that grow from
 * tokens_before[r] to tokens_after[r] cached tokens (negative counts as 0; a
 * request that shrinks does not move).  Request r needs
 *   ceil(after / page_size) - ceil(before / page_size)
 * pages; they are taken from free_pages[free_begin ..) in request order and
 * written to page_table[r][ceil(before / page_size) ..); entries of pages
 * already held are left alone.  free_end[0] receives the place of the first
 * page not taken.  token_base[r] receives the number of new tokens of the
 * requests before r, token_base[n_requests] their sum (the row base of each
 * request in a packed batch of new tokens); slots[token_base[r] + i] the pool
 * slot page * page_size + offset of new token i of request r, and every entry
 * of slots past the sum -1.
 * Where the free list ends the remaining entries are -1, as are the slots in
 * them (KAMERA_STATUS_NO_PAGE); a page number outside the pool gives -1
 * (KAMERA_STATUS_BAD_PAGE); a request is cut at pt_stride pages
 * (KAMERA_STATUS_BAD_LENGTH), and its further tokens have no slot entry.
 * No output may overlap an input or another output, except that page_table is
 * both. */
typedef struct {
  int32_t n_requests;            /* 0 .. KAMERA_MAX_REQUESTS                   */
  int32_t page_size;             /* > 0; n_requests * pt_stride * page_size    */
  int32_t pt_stride;             /*   must be below 2^31                       */
  int32_t n_pool_pages;
  const int32_t* tokens_before;  /* device [n_requests], or NULL = 0           */
  const int32_t* tokens_after;   /* device [n_requests]                        */
  const int32_t* free_pages;     /* device [n_free]                            */
  int32_t n_free;
  const int32_t* free_begin;     /* device [1], or NULL = 0                    */
  int32_t* free_end;             /* device [1]                                 */
  int32_t* page_table;           /* device [n_requests][pt_stride]             */
  int32_t* token_base;           /* device [n_requests + 1]                    */
  int64_t* slots;                /* device [n_slots], or NULL                  */
  int64_t n_slots;
  uint32_t* status;
} kamera_page_tables_args;

/* kamera_append_paged8 -- n = chunk_tokens[c] (n_tokens if NULL) bf16 K and V
 * rows of every chunk c and layer into the 8-bit cache, behind the
 * tokens_before[c] (0 if NULL) tokens that the chunk's pages hold already:
 * row i becomes token tokens_before[c] + i, in page page_table[c][token /
 * page_size].  Rows are read as in kamera_shift: token i of chunk c at
 *   k + c*k_stride[0] + l*k_stride[1] + (row_base[c] + i)*k_stride[2]
 *     + h*k_stride[3]                                   (row_base NULL = 0).
 * A page that receives rows takes the exponent e of its new rows' largest
 * finite magnitude; a page that held tokens before keeps its own where that
 * is larger, and is otherwise brought to the new one (bytes rounded to
 * nearest even where they leave the normal range).  Elements are rounded to
 * the nearest e4m3 value, ties to even; infinities and NaN are stored as NaN
 * and take no part in e.  Slots past the last token are not written.  Tokens
 * past the pages of a row (pt_pages) are left out (KAMERA_STATUS_BAD_LENGTH).
 *
 * k_sum (with k_sum_scale; both or neither): when a page is filled, the sum
 * of its page_size keys, column by column, as int8 with one power-of-two
 * scale: t = sum of the bytes' values (NaN counts as 0; exact in fp32),
 * f the least exponent (>= -100) with max |t| <= 127 * 2^f,
 *   k_sum[j] = round(t[j] * 2^-f) (ties to even), k_sum_scale = scale * 2^f
 * (fp32: 0 for a page of zeros).
 * kamera_select_pages scores pages by it.
 * A page may receive rows of one chunk only.  No output may overlap an input
 * (checked on the extents that the sizes imply) or another output. */
typedef struct {
  int32_t n_chunks;
  int32_t n_layers;
  int32_t n_heads;               /* KV heads                                   */
  int32_t head_dim;              /* 64 or 128                                  */
  int32_t n_tokens;              /* most new tokens of a chunk                 */
  int32_t page_size;             /* 16, 32 or 64                               */
  int32_t pt_stride;
  int32_t n_pool_pages;
  const int32_t* chunk_tokens;   /* device [n_chunks], or NULL                 */
  const int32_t* tokens_before;  /* device [n_chunks], or NULL                 */
  const int32_t* row_base;       /* device [n_chunks], or NULL                 */
  const int32_t* page_table;     /* device [n_chunks][pt_stride], pt_pages of  */
                                 /*   each row in use                          */
  const void* k;
  int64_t k_stride[4];           /* chunk, layer, row, head                    */
  const void* v;
  int64_t v_stride[4];
  void* k_cache;
  int64_t k_cache_stride[4];     /* layer, page, token, head                   */
  void* v_cache;
  int64_t v_cache_stride[4];
  float* k_scale;
  int64_t k_scale_stride[3];     /* layer, page, head                          */
  float* v_scale;
  int64_t v_scale_stride[3];
  int8_t* k_sum;                 /* optional                                   */
  int64_t k_sum_stride[3];       /* layer, page, head (multiples of 16)        */
  float* k_sum_scale;
  int64_t k_sum_scale_stride[3];
  uint32_t* status;
  int32_t pt_pages;              /* entries of a page-table row (0: pt_stride) */
} kamera_append_args;

/* kamera_select_pages -- for one query token a request and every KV head, the
 * n_keep pages of the request (of the first ceil(kv_tokens / page_size)) that
 * matter most, as ascending page indices into its page-table row; fewer, where
 * the request has fewer.  sel[r][h][0 .. sel_count[r][h]) receives them, the
 * rest of the n_keep entries -1.  The first n_first and the last n_last pages
 * are always among them (the last one need not be full); the others are ranked
 * by
 *   score(p) = (max over the group's query heads g of
 *               sum_j q8[g][j] * k_sum[p][h][j]) * k_sum_scale[p][h],
 * ties to the lower index.  q8 is the group's query rows as int8 with one
 * power-of-two scale: round(q * 2^-f), ties to even, f the least exponent
 * (>= -100) at which the group's largest finite magnitude is at most 127 * 2^f;
 * what is not finite counts as 0.  The integer sums are exact, so the
 * selection is one answer, whatever computes it.  A page number outside the
 * pool is flagged and its page ranked last, as is a page whose score is not a
 * number; a request of at most n_keep pages keeps them all, without a look at
 * their numbers. */
typedef struct {
  int32_t n_requests;
  int32_t n_q_heads;             /* a multiple of n_kv_heads; group <= 64      */
  int32_t n_kv_heads;
  int32_t head_dim;              /* 64 or 128                                  */
  int32_t n_keys;                /* most cached tokens of a request            */
  int32_t page_size;
  int32_t pt_stride;
  int32_t n_pool_pages;
  const int32_t* kv_tokens;      /* device [n_requests], at most n_keys        */
  const int32_t* page_table;     /* device [n_requests][pt_stride]             */
  const void* q;                 /* bf16, request r, head g at                 */
  int64_t q_stride[2];           /*   q + r*q_stride[0] + g*q_stride[1]        */
  const int8_t* k_sum;
  int64_t k_sum_stride[2];       /* page, head                                 */
  const float* k_sum_scale;
  int64_t k_sum_scale_stride[2];
  int32_t n_keep;                /* >= n_first + n_last                        */
  int32_t n_first;               /* >= 0                                       */
  int32_t n_last;                /* >= 1                                       */
  int32_t* sel;                  /* device [n_requests][n_kv_heads][n_keep]    */
  int32_t* sel_count;            /* device [n_requests][n_kv_heads]            */
  void* workspace;               /* as in kamera_attend_args                   */
  int64_t workspace_bytes;       /* at least kamera_select_workspace(args)     */
  uint32_t* status;
} kamera_select_args;

typedef enum {
  KAMERA_CACHE_BF16 = 0,         /* the pool that kamera_rehydrate writes      */
  KAMERA_CACHE_E4M3 = 1          /* the 8-bit cache of kamera_append_paged8    */
} kamera_cache_type;

/* kamera_attend_paged -- softmax attention of a batch of requests over one
 * layer of the paged cache.  Request r has n = q_tokens[r] (n_queries if NULL)
 * query tokens, rows q_base[r] + i (r*n_queries + i if NULL) of q and out, and
 * kv = kv_tokens[r] tokens in the cache, its queries' own included.  Query
 * head g reads KV head g / (n_q_heads / n_kv_heads):
 *   out[i][g] = sum_t p[t] V[t],  p = softmax over the seen t of
 *               scale * <q[i][g], K[t]>,
 * where query i sees the keys t in [0, kv), with causal = 1 those with
 * t <= kv - n + i, and with window > 0 (causal only) of these the last
 * `window`.  A row that sees no key gets 0 (and lse = -infinity), and so does
 * one whose every score is -infinity.  What a row does not see does not touch
 * it, whatever it holds.  lse (optional, fp32)
 * receives the natural logarithm of sum exp(scale * <q, K[t]>) at
 * lse + row*lse_stride[0] + g*lse_stride[1]; with it, results over parts of a
 * context can be joined.
 * Scores, softmax statistics and sums are fp32; p is rounded to bf16 for the
 * product with V, the output once to bf16.
 *
 * sel (optional; n_queries must be 1): only the pages sel[r][h][0 ..
 * sel_count[r][h]) (indices into the page-table row, as kamera_select_pages
 * writes them) are read.
 * Keys in pages whose number is outside the pool are not seen (and flagged),
 * nor are selected pages past the pages of a row (pt_pages).
 *
 * Work is split over the keys where there are few rows: n_splits parts a row
 * (0: chosen from the sizes), joined by a second kernel on the same stream.
 * workspace then holds the parts: device memory of at least
 * kamera_attend_workspace(args) bytes, 16-byte aligned, not used by other work
 * at the same time; its contents need not be kept or cleared.
 * Outputs must not overlap inputs, the workspace or each other. */
typedef struct {
  int32_t n_requests;
  int32_t n_q_heads;             /* a multiple of n_kv_heads; group <= 64      */
  int32_t n_kv_heads;
  int32_t head_dim;              /* 64 or 128                                  */
  int32_t n_queries;             /* most query tokens of a request             */
  int32_t n_keys;                /* most cached tokens of a request            */
  int32_t page_size;             /* a multiple of 16                           */
  int32_t pt_stride;
  int32_t n_pool_pages;
  int32_t cache_type;            /* kamera_cache_type                          */
  int32_t causal;                /* 1 or 0                                     */
  int32_t window;                /* > 0: keys seen at most; 0: all             */
  float scale;                   /* finite                                     */
  int32_t n_splits;              /* 0: automatic; else 1 .. 512                */
  const int32_t* q_tokens;       /* device [n_requests], or NULL               */
  const int32_t* q_base;         /* device [n_requests], or NULL               */
  const int32_t* kv_tokens;      /* device [n_requests], at most n_keys        */
  const int32_t* page_table;     /* device [n_requests][pt_stride], pt_pages   */
                                 /*   of each row in use                       */
  const void* q;                 /* bf16                                       */
  int64_t q_stride[2];           /* row, head                                  */
  void* out;                     /* bf16                                       */
  int64_t out_stride[2];
  float* lse;
  int64_t lse_stride[2];
  const void* k_cache;
  int64_t k_cache_stride[3];     /* page, token, head                          */
  const void* v_cache;
  int64_t v_cache_stride[3];
  const float* k_scale;          /* E4M3 only                                  */
  int64_t k_scale_stride[2];     /* page, head                                 */
  const float* v_scale;
  int64_t v_scale_stride[2];
  const int32_t* sel;            /* optional: device [n_requests][n_kv_heads]  */
  const int32_t* sel_count;      /*   [sel_stride], and their counts           */
  int32_t sel_stride;
  int32_t pt_pages;              /* entries of a page-table row (0: pt_stride) */
  void* workspace;
  int64_t workspace_bytes;
  uint32_t* status;
} kamera_attend_args;

int kamera_page_tables(const kamera_page_tables_args* args, void* stream);
int kamera_append_paged8(const kamera_append_args* args, void* stream);
int kamera_select_pages(const kamera_select_args* args, void* stream);
int kamera_attend_paged(const kamera_attend_args* args, void* stream);

/* Bytes of workspace that kamera_attend_paged and kamera_select_pages need for
 * `args` (its pointers are not looked at, workspace and workspace_bytes
 * included), 0 where the work is not split; or the negative error code of a
 * refused size. */
int64_t kamera_attend_workspace(const kamera_attend_args* args);
int64_t kamera_select_workspace(const kamera_select_args* args);

/* As kamera_validate, for the entry points above: 0 kamera_page_tables,
 * 1 kamera_append_paged8, 2 kamera_select_pages, 3 kamera_attend_paged. */
int kamera_validate_cache(int32_t which, const void* args);

/* Host-side check of a page table copy (host memory, n_chunks x pt_stride,
 * the first ceil(tokens/page_size) entries of each row are used): every used
 * entry in [0, n_pool_pages) and no page used twice.  Returns KAMERA_OK or
 * KAMERA_ERR_RANGE (out of range) / KAMERA_ERR_ALIAS (duplicate). */
int kamera_check_page_table(const int32_t* host_page_table, int32_t n_chunks,
                            int32_t pt_stride, int32_t n_tokens,
                            int32_t page_size, int32_t n_pool_pages);

/* Run exactly the host-side checks of an entry point (0 kamera_rehydrate,
 * 1 kamera_shift, 2 kamera_scatter_paged, 3 kamera_gather_paged,
 * 4 kamera_form_patch) on `args` without launching anything: KAMERA_OK when
 * the call would be enqueued, else the error code the call would return.
 * Touches no device memory. */
int kamera_validate(int32_t which, const void* args);

/* Which kernel kamera_rehydrate would launch for `args` (see
 * kamera_kernel_choice), after exactly its host-side checks:
 * KAMERA_PLAN_PER_HEAD, KAMERA_PLAN_ROW_GROUP (8 heads per workgroup),
 * KAMERA_PLAN_ROW_GROUP4 (4 heads per workgroup), KAMERA_PLAN_NONE for a call
 * with nothing to do, or the negative error code the call would return.  A
 * positive plan equals the kamera_kernel_choice that requests that kernel.
 * Touches no device memory. */
#define KAMERA_PLAN_NONE 0
#define KAMERA_PLAN_PER_HEAD 1
#define KAMERA_PLAN_ROW_GROUP 2
#define KAMERA_PLAN_ROW_GROUP4 3
int kamera_rehydrate_plan(const kamera_rehydrate_args* args);

/* How the row-group kernel would spread a kamera_rehydrate call for `args`
 * (see kamera_row_schedule), after exactly its host-side checks:
 * KAMERA_SCHEDULE_PERSISTENT or KAMERA_SCHEDULE_BLOCKS; 0 when the call runs
 * the per-head kernel or has nothing to do; else the negative error code the
 * call would return.  Touches no device memory. */
int kamera_rehydrate_schedule(const kamera_rehydrate_args* args);

/* Text of the last error on the calling thread ("" after a successful call);
 * valid until the next call on that thread. */
const char* kamera_last_error(void);
int kamera_abi_version(void);
/* sizeof of the argument structs: 0 rehydrate, 1 shift, 2 scatter, 3 plane,
 * 4 rope, 5 form, 6 page tables, 7 append, 8 select, 9 attend; -1 otherwise.  Lets a foreign-function binding check its
 * layout. */
int64_t kamera_struct_size(int32_t which);

#ifdef __cplusplus
}
#endif

#endif /* KAMERA_H */
