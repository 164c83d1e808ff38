/*
 * libcdb, verification of drafted tokens: several guessed tokens per sequence
 * run through the stage operators of libcdb.h in one pass, as a tree of
 * alternatives over the sequence's paged, depth-indexed K/V cache.
 *
 * One round of a serving loop, all on the device and on one stream:
 *   cdb_map_pages      pages for every sequence's committed and drafted positions
 *   cdb_tree_rows      the drafted trees as the rows of one stage call
 *   cdb_tree_prelude, cdb_tree_step, cdb_tree_coda
 *                      the stage calls, with cdb_tree_attention in every layer
 *   cdb_tree_accept    the path of drafted tokens that the model would have
 *                      produced itself (greedy), and the token that follows it,
 *   or cdb_tree_sample a path and a token that are distributed as the model's own
 *                      samples
 *   cdb_tree_commit    the K/V of that path moved to the positions it takes
 *   cdb_map_pages      the pages behind it given back
 *
 * A tree of n nodes over a sequence with `len` committed positions keeps the
 * K/V of node j at cache position len + j, in every plane, while its RoPE
 * position is len + depth(j) (a root: len).  Node j sees positions 0..len - 1,
 * its ancestors and itself.  Parents come before their children.
 *
 * The conventions of libcdb.h hold: caller-owned buffers, everything enqueued
 * on the given stream, nothing allocated or synchronised, sticky device errors
 * in the workspace (cdb_read_device_error).  A workspace of
 * cdb_tree_workspace_bytes serves every call below, and those of libcdb.h.
 * Calls on one workspace must not overlap.
 */
#ifndef LIBCDB_TREE_H
#define LIBCDB_TREE_H

#include "libcdb.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CDB_TREE_MAX_NODES 64  /* nodes of one tree */
#define CDB_TREE_MAX_TREES 256 /* trees of one call */

/* Device error code beside those of libcdb.h: cdb_map_pages found too few free
 * pages (or a stack too small for those given back) and changed nothing. */
enum { CDB_DEV_NO_PAGES = 4 };

/* What a row of drafted tokens sees, beside cdb_rows (device arrays of n_rows
 * entries; those past a device row count do not matter).
 *   base      committed positions of the row's sequence: 0..base - 1 are visible
 *   mask      bit j: cache position base + j is visible too (its own included)
 *   rope_pos  the position the row's token stands at (RoPE); cdb_rows.pos is the
 *             cache position that receives its K/V
 * Rows may come in any order and sit at any loop index.  Adjacent rows of one
 * sequence, plane and base are read together (K/V once for all of them), so a
 * tree's rows belong next to each other.  max_nodes (host, 1..64): the most rows
 * expected next to each other of one tree; it picks launch shapes, results do
 * not depend on it.  A row's result does not depend on the other rows. */
typedef struct {
    int32_t max_nodes;
    const int32_t* base;
    const uint64_t* mask;
    const int32_t* rope_pos;
} cdb_tree;

/* Workspace of the calls below for up to max_rows rows (at most 256) and
 * max_seqs sequences (which need no room of their own); 0 if unsupported.  At
 * least cdb_workspace_bytes(desc, max_rows).  Cleared once by
 * cdb_workspace_init. */
size_t cdb_tree_workspace_bytes(const cdb_model_desc* desc, int32_t max_rows, int32_t max_seqs);

/* The free pages of one pool, a stack in device memory: free_ids[0 ..
 * *free_count - 1], the next page on top (the highest index); capacity entries. */
typedef struct {
    int32_t* free_ids;
    int32_t* free_count;
    int32_t capacity;
} cdb_page_pool;

/* Brings every sequence's mapped pages to what len[s] positions need: pages
 * ceil(len[s] / 16) .. mapped[s] - 1 are given back and unmapped (-1), pages
 * mapped[s] .. ceil(len[s] / 16) - 1 are taken and mapped, in every plane of
 * every stage that has layers; then mapped[s] is the new count.  len[s] < 0
 * leaves sequence s as it is.
 *   page_table  device int32 [max_seqs][r_max + 2][max_pages], as cdb_kv has it
 *   len, mapped device int32 [max_seqs]
 *   kv_layout   CDB_KV_FULL, CDB_KV_SHARED or CDB_KV_FIRST_THEN_SHARED
 *               (libcdb_driver.h): which core planes share a page
 *   pre, core, coda  the pools of the stages with layers (others are not read),
 *               each with a stack of its own
 * First the given-back pages go onto each stack, the last in (sequence, page,
 * plane) order first; then new ones come off it in (sequence, page, plane)
 * order.  Cutting a sequence back right after growing it so restores the stack.
 * A stack's entries from its count on keep what stood there last.  All or
 * nothing: if a pool has too few pages (or its stack too few entries), a length
 * needs more than max_pages pages, or mapped or a count is out of range, nothing
 * changes and the workspace's error code is set (CDB_DEV_NO_PAGES,
 * CDB_DEV_BAD_INDEX).  If a page id among those given back or taken is negative,
 * nothing that is mapped or free changes (CDB_DEV_UNMAPPED_PAGE); pages that were
 * to be mapped read -1 then, and stack entries from the count on are lost. */
cdb_status cdb_map_pages(const cdb_model_desc* desc, int32_t* page_table, int32_t max_seqs, int32_t max_pages,
                         const cdb_page_pool* pre, const cdb_page_pool* core, const cdb_page_pool* coda,
                         int32_t kv_layout, const int32_t* len, int32_t* mapped, void* ws, size_t ws_bytes,
                         hipStream_t stream);

/* Drafted trees (device arrays; the counts are host values):
 *   seq       [n_trees] sequence of each tree, each at most once
 *   len       [max_seqs] committed positions, by sequence
 *   n_nodes   [n_trees] nodes of each tree, 0..max_nodes
 *   parent    [n_trees][max_nodes] node index of each node's parent in its tree
 *             (smaller than its own), -1 for a root
 *   tokens    [n_trees][max_nodes] drafted token ids
 * 1 <= max_nodes <= 64, 0 <= n_trees <= 256. */
typedef struct {
    int32_t n_trees, max_nodes, max_seqs;
    const int32_t* seq;
    const int32_t* len;
    const int32_t* n_nodes;
    const int32_t* parent;
    const int32_t* tokens;
} cdb_drafts;

/* Rows of drafted trees, packed in (tree, node) order (device, `capacity`
 * entries): the arrays of cdb_rows and cdb_tree, the input tokens, row0
 * [n_trees] = each tree's first row, n_rows [1] = the row count (for
 * cdb_rows.d_n_rows).  Entries from n_rows on are left as they were. */
typedef struct {
    int32_t capacity;
    int32_t* row0;
    int32_t* n_rows;
    int32_t* seq;
    int32_t* pos;
    int32_t* base;
    int32_t* rope_pos;
    int32_t* tokens;
    uint64_t* mask;
} cdb_row_map;

/* Lays the trees out as rows.  A tree with a bad count, sequence or length, or
 * of a sequence that an earlier tree has, gets no rows (its row0 is that of the
 * next tree's first row, as for a tree of no nodes), and a parent that is not
 * an earlier node of the tree makes its node a root; either sets
 * CDB_DEV_BAD_INDEX.  Trees from the first on that does not fit into `capacity`
 * get no rows, row0 = -1 and the same code. */
cdb_status cdb_tree_rows(const cdb_drafts* drafts, const cdb_row_map* out, void* ws, size_t ws_bytes,
                         hipStream_t stream);

/* Attention of drafted rows in one layer, beside cdb_paged_attention (same q,
 * out and stage / layer arguments): row i attends to the positions that
 * tree->base[i] and tree->mask[i] name, in its own plane.  Reads the cache only;
 * the rows' own K/V must be in it.  What a masked position holds (NaN included)
 * does not reach a row.  What a row sees may be infinite or NaN, and its scores and
 * sums as large as 32 bits hold: it gets what softmax and sum give then, at a slower
 * pace.  A row that sees nothing gets zeros.  The stage's pool
 * has at least one page, however few are mapped.  A row whose
 * sequence, loop index or positions are out of range is skipped
 * (CDB_DEV_UNMAPPED_PAGE), an unmapped page is left out (the same code). */
cdb_status cdb_tree_attention(const cdb_model_desc* desc, const cdb_kv* kv, const cdb_rows* rows,
                              const cdb_tree* tree, int32_t stage, int32_t layer, const float* q, void* out, void* ws,
                              size_t ws_bytes, hipStream_t stream);

/* The stage calls of libcdb.h over drafted rows: cdb_boundary_prelude,
 * cdb_loop_step (gate NULL) or cdb_loop_step_gated, cdb_boundary_coda, with
 * RoPE at tree->rope_pos and the attention of cdb_tree_attention.  Everything
 * else is as there, K/V writes and copy-on-exit at rows->pos included. */
cdb_status cdb_tree_prelude(const cdb_model* model, const cdb_kv* kv, const cdb_state* state, const cdb_rows* rows,
                            const cdb_tree* tree, const int32_t* tokens, void* ws, size_t ws_bytes,
                            hipStream_t stream);
cdb_status cdb_tree_step(const cdb_model* model, const cdb_kv* kv, const cdb_state* state, const cdb_rows* rows,
                         const cdb_tree* tree, const cdb_gate* gate, const cdb_step_out* out, void* ws,
                         size_t ws_bytes, hipStream_t stream);
cdb_status cdb_tree_coda(const cdb_model* model, const cdb_kv* kv, const cdb_state* state, const cdb_rows* rows,
                         const cdb_tree* tree, float* logits, int32_t* next_ids, void* ws, size_t ws_bytes,
                         hipStream_t stream);

/* Greedy acceptance, and what cdb_tree_commit takes (device):
 *   path  int32 [n_trees][max_nodes] accepted nodes from the root down, then -1
 *   count int32 [n_trees] how many
 *   next  int32 [n_trees] the greedy id that follows them */
typedef struct {
    int32_t* path;
    int32_t* count;
    int32_t* next;
} cdb_accepted;

/* Walks down each tree as long as a child is what the model says: at first a
 * root with token first_ids[t] (int32 [n_trees], the greedy id after the
 * committed positions), then a child whose token is next_ids[row0[t] + node]
 * (next_ids int32 [n_rows], by row, as the coda writes it); of several the one
 * with the lowest index.  row0: as cdb_tree_rows wrote it (-1: the tree has no
 * rows, nothing is accepted).  A node whose parent is not an earlier node is never
 * reached, and one whose row is outside [0, n_rows) neither (CDB_DEV_BAD_INDEX).
 * n_nodes, parent and tokens of `drafts` are read, and seq and len unless they are
 * NULL: of a tree that cdb_tree_rows gives no rows because of its sequence, length
 * or count nothing is accepted (CDB_DEV_BAD_INDEX, a bad count aside).  Without
 * them the caller sees to it that every tree with nodes and a row0 >= 0 has rows. */
cdb_status cdb_tree_accept(const cdb_drafts* drafts, const int32_t* row0, const int32_t* next_ids, int32_t n_rows,
                           const int32_t* first_ids, const cdb_accepted* out, void* ws, size_t ws_bytes,
                           hipStream_t stream);

/* Device error code beside those above: logits that are no distribution (a NaN, an infinity
 * that is not -inf, or nothing else than -inf), or a temperature that is not above 0 and finite. */
enum { CDB_DEV_BAD_VALUE = 5 };

#define CDB_SAMPLE_MAX_VOCAB (1 << 20)

/* What sampled acceptance reads beside the trees (device):
 *   logits         fp32, row r at logits + r * logits_stride: the target's after every
 *                  drafted node, by row, as the coda writes them
 *   draft_logits   the drafter's after every node, likewise: those that the node's children
 *                  were drawn from, each by itself.  NULL: the drafter was sure of each
 *                  token that it guessed (probability 1)
 *   *_stride       in values, at least the model's vocab, a multiple of 4; the logits'
 *                  addresses are multiples of 16
 *   temperature, draft_temperature   fp32 [n_trees], above 0 and finite: the probabilities are
 *                  softmax(logits / temperature); NULL: 1
 *   u_node         fp32 [n_trees][max_nodes] random numbers, even in [0, 1), one per node
 *   u_next         fp32 [n_trees] one per tree, for the token that follows
 * -inf among the logits is a probability of 0 (tokens that are masked out). */
typedef struct {
    const float* logits;
    const float* draft_logits;
    int64_t logits_stride, draft_stride;
    const float* temperature;
    const float* draft_temperature;
    const float* u_node;
    const float* u_next;
} cdb_sampling;

/* Sampled acceptance: the accepted tokens and `next` are distributed as if each had
 * been drawn from the target's probabilities in turn, whatever the drafter's are.  Walks down
 * each tree: at first to the lowest root with token first_ids[t] (int32 [n_trees], the
 * token already drawn after the committed positions; none: nothing is accepted and next is
 * that token).  At a node with target p and drafter q, r = p; for its children in
 * order, with token x and u of u_node:
 *   u q(x) < r(x):  the child is accepted, and the walk goes on there;
 *   otherwise       r <- max(r - q, 0), divided by its sum (a sure drafter: r without x,
 *                   divided by its sum; if nothing is left, r stays).
 * When no child is left, next is the first token whose cumulated r, from token 0 on, is above
 * u_next times the sum of r.  Probabilities and sums are in 64 bits.
 * The trees, row0, n_rows (at most 256 here) and `out` are as for cdb_tree_accept, with the
 * same refusals; no row belongs to two trees; a drafted token outside [0, vocab) is not accepted (CDB_DEV_BAD_INDEX).
 * A walk that comes to logits that are no distribution ends there, next = -1
 * (CDB_DEV_BAD_VALUE); a tree with a bad temperature accepts nothing (the same code). */
cdb_status cdb_tree_sample(const cdb_model_desc* desc, const cdb_drafts* drafts, const int32_t* row0, int32_t n_rows,
                           const int32_t* first_ids, const cdb_sampling* sampling, const cdb_accepted* out, void* ws,
                           size_t ws_bytes, hipStream_t stream);

/* Moves the K/V of each tree's accepted nodes from cache position len + path[i]
 * to len + i, in every layer and plane of every stage (planes that share their
 * pages once), so that the context goes on without gaps.  No other sequence maps
 * the pages of these positions.  accepted->next is not
 * read; `drafts` needs seq and len only.  The caller then adds count to len.  A
 * path that is not increasing or not in [0, max_nodes), a sequence out of range
 * or given twice (the later tree) and planes that share some but not all pages
 * of the moved positions are left as they are (CDB_DEV_BAD_INDEX), and so is a
 * plane with an unmapped page there (CDB_DEV_UNMAPPED_PAGE). */
cdb_status cdb_tree_commit(const cdb_model_desc* desc, const cdb_kv* kv, const cdb_drafts* drafts,
                           const cdb_accepted* accepted, void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
