/*
 * libcdb, chunks of new tokens: the attention half of a layer for the new tokens
 * of several sequences at once, over the paged, depth-indexed K/V cache of
 * libcdb.h.  A chunk is one to thousands of consecutive positions of one
 * sequence: a decoded token, a drafted chain, a prompt or a part of one.
 *
 *   cdb_chunk_qkv        queries and keys normalised head by head (optional) and
 *                        rotated to their positions, keys and values written to
 *                        the cache, queries to a buffer
 *   cdb_chunk_attention  causal attention of the chunks' rows over the cache
 *
 * Both serve programs that run their projections themselves, next to
 * cdb_paged_attention and cdb_tree_attention (which read the same cache), for
 * calls of more rows than those take.
 *
 * The conventions of libcdb.h hold: caller-owned buffers, everything enqueued
 * on the given stream, nothing allocated or synchronised, sticky device errors
 * in the workspace (cdb_read_device_error).  Calls on one workspace must not
 * overlap.
 */
#ifndef LIBCDB_CHUNK_H
#define LIBCDB_CHUNK_H

#include "libcdb.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CDB_MAX_CHUNKS 256       /* chunks of one call */
#define CDB_MAX_CHUNK_ROWS 65536 /* rows of one call, all chunks together */

/* Types of values that a call takes in either form. */
enum { CDB_F32 = 0, CDB_BF16 = 1 };

/* Orders of an output of n rows of d bf16 values. */
enum {
    CDB_ORDER_FRAGMENTS = 0, /* as cdb_paged_attention writes it, rows rounded up to 32 */
    CDB_ORDER_ROWS = 1       /* row-major [n_rows][d] */
};

/* The chunks of a call (device arrays; the counts are host values):
 *   row0   int32 [n_chunks + 1], not decreasing, from 0 or more to n_rows or less:
 *          chunk i has rows row0[i] .. row0[i + 1] - 1 (there may be none)
 *   seq    int32 [n_chunks] sequence of each chunk (several may be of one)
 *   pos0   int32 [n_chunks] position of its first row; the others follow
 *   c      int32 [n_chunks] loops completed: the core plane is c + 1 (read for
 *          the core only, may be NULL otherwise)
 * n_rows (host) is what the row buffers hold; rows outside every chunk are
 * neither read nor written, so one captured call replays for any chunks that
 * fit into its n_chunks and n_rows.
 * A row0 that decreases or leaves 0..n_rows refuses the whole call: nothing is
 * written but the error code, CDB_DEV_BAD_INDEX.  A chunk whose sequence, loop or
 * positions are out of range is skipped with the same code. */
typedef struct {
    int32_t n_chunks, n_rows;
    const int32_t* row0;
    const int32_t* seq;
    const int32_t* pos0;
    const int32_t* c;
} cdb_chunks;

/* Workspace of both calls for up to max_rows rows in up to max_chunks chunks; 0 if
 * unsupported.  Cleared once by cdb_workspace_init. */
size_t cdb_chunk_workspace_bytes(const cdb_model_desc* desc, int32_t max_rows, int32_t max_chunks);

/* Queries, keys and values as the projections left them (device): row r of q is at
 * q + r * q_stride values, its heads one after another; k and v likewise, so the
 * parts of a fused [n_rows][3 d] are given by their first values and stride 3 d.
 *   type      CDB_F32 or CDB_BF16, of all three
 *   *_stride  in values, at least d, a multiple of 16 bytes; so are the addresses
 *   norm      1: every head of q and k is first divided by its root mean square,
 *             sqrt(mean(x^2) + desc->rms_eps), and multiplied by the gains
 *   q_gain, k_gain   bf16 [head_dim], NULL: gains of 1 (not read without norm)
 *   rope_pos  int32 [n_rows] positions to rotate to where they are not the rows'
 *             own, NULL: they are */
typedef struct {
    const void* q;
    const void* k;
    const void* v;
    int32_t type;
    int32_t norm;
    int64_t q_stride, k_stride, v_stride;
    const void* q_gain;
    const void* k_gain;
    const int32_t* rope_pos;
} cdb_qkv;

/* For every row: q and k normalised (norm) and rotated, value j of a head with value
 * j + head_dim / 2 by the angle position * rope_base^(-2 j / head_dim); k and v
 * rounded to bf16 and written to the cache at the row's position, in its plane of
 * stage `stage` (0 prelude, 1 core -> plane c + 1, 2 coda), layer `layer`; q written
 * to q_out [n_rows][d] as q_type (CDB_F32, CDB_BF16), which may be in->q itself where
 * types and strides (d) are the same, and otherwise lies apart from q, k and v; all of
 * them lie apart from the stage's pool (CDB_ERR_INVALID_ARG).  Arithmetic and norms are in 32 bits, angles in
 * 64.  A position of a plane belongs to one row of the call.  A row whose page is
 * not mapped writes q only (CDB_DEV_UNMAPPED_PAGE). */
cdb_status cdb_chunk_qkv(const cdb_model_desc* desc, const cdb_kv* kv, const cdb_chunks* chunks, int32_t stage,
                         int32_t layer, const cdb_qkv* in, void* q_out, int32_t q_type, void* ws, size_t ws_bytes,
                         hipStream_t stream);

/* Causal attention: the row at position p of a chunk attends to positions 0..p of its
 * sequence in the chunk's plane,
 *   out[i][h] = softmax_s(q[i][h] . K_s / sqrt(head_dim)) V_s,
 * rounded to bf16.  q: [n_rows][d] of q_type; out: in the given order, apart from q and the stage's pool, rows outside
 * every (good) chunk left as they were.  Reads the cache only; the rows' own K/V must be in it.
 * With CDB_BF16 queries the weights are rounded to bf16 for the product with V; with
 * CDB_F32 both are taken in two bf16 parts (about 16 bits).  Sums and statistics are in 32
 * bits.
 * What a row may not see (NaN included) does not reach it.  q and the K and V that rows see
 * are finite, and so are their scores and sums in 32 bits; where they are not, the rows that
 * see them get no number or an infinity, and no other row changes.  Only a score of -inf
 * may also count as that of a key that is not there.  An unmapped page is
 * left out (CDB_DEV_UNMAPPED_PAGE); a row that sees nothing gets zeros.  The stage's pool has
 * at least one page, however few are mapped.
 * A chunk's result does not depend on the other chunks; n_rows, n_chunks and the table's
 * max_pages choose how contexts are split, so roundings may differ between calls of
 * different ones.  The same call gives the same bits. */
cdb_status cdb_chunk_attention(const cdb_model_desc* desc, const cdb_kv* kv, const cdb_chunks* chunks, int32_t stage,
                               int32_t layer, const void* q, int32_t q_type, void* out, int32_t out_order, void* ws,
                               size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
