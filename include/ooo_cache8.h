/*
 * ooo_cache8.h - entry points of libooo for a batch whose cache pages hold
 * 8-bit numbers, and for sequences that continue another one's cache.
 *
 *   ooo_paged_append8    q/k norms and rotation of a batch's new rows, q out,
 *                        k/v quantised into the sequences' pages
 *   ooo_paged_plan8      the split of a batch's attention work, once a step
 *   ooo_paged_attn8      attention over the shared prompt, each sequence's own
 *                        pages and its ancestors among the new rows
 *   ooo_paged_compact8   moves the accepted rows of every sequence together
 *   ooo_paged_fork, ooo_paged_fork8
 *                        sequences become continuations of others: whole pages
 *                        are shared, the open one is copied
 *
 * The conventions of ooo.h and the batch of ooo_batch.h hold.  A pool's
 * elements are e4m3 numbers (OCP: a sign, four bits of exponent, three of
 * fraction; no infinities), one byte each.  Blocks of 32 consecutive rows of a
 * page share one scale for each KV head, K and V apart: the byte E stands for
 * 2^(E - 127), and an element for its number times that.  Scales go from 2^-100
 * to 2^119 (the entry points write no other and read these).  An append takes the
 * least one that brings the values of the rows that it puts into a block to at
 * most 448, drafts that are rejected later among them; a commit the largest of the
 * blocks that its rows come from; and it never falls while the block holds
 * committed rows.  So a scale is an upper bound for what its block holds.  A power
 * of two, so that a scale that is larger than these rows need, or that grows under
 * them, costs them nothing but the last bits of numbers that become subnormal:
 * values below 2^(E - 127 - 6) are multiples of 2^(E - 127 - 9), and a cache filled
 * through rejected drafts may differ in them from one that never saw these.
 *
 * In an ooo_paged_batch for these entry points page_rows is at least 32 and
 * page_stride counts bytes (a multiple of 16); dt is the type of q, qkv, the
 * norms and out.
 */
#ifndef OOO_CACHE8_H
#define OOO_CACHE8_H

#include "ooo_batch.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ooo_cache8 - the pools of n_layers layers.  The struct lives in HOST memory,
 * the pools in DEVICE memory.
 *   k_pages, v_pages     [n_layers][n_pages] pages [n_kv_heads][page_rows]
 *                        [head_dim] of e4m3 (16-byte aligned)
 *   k_scales, v_scales   [n_layers][n_pages][n_kv_heads][page_rows / 32] bytes
 *   layer_stride         bytes from one layer's pages to the next's (a
 *                        multiple of 16)
 *   scale_stride         bytes from one page's scales to the next's, at least
 *                        n_kv_heads * page_rows / 32
 *   scale_layer_stride   bytes from one layer's scales to the next's
 */
typedef struct {
  void* k_pages;
  void* v_pages;
  void* k_scales;
  void* v_scales;
  int64_t layer_stride;
  int64_t scale_stride;
  int64_t scale_layer_stride;
  int32_t n_layers;
} ooo_cache8;

/*
 * ooo_paged_append8 - as ooo_paged_append, with k and v rounded once, from
 * float32, to the nearest e4m3 number under their block's scale (ties to even).
 * The scale of a block that new rows of a sequence lie in is what they need,
 * and where the block holds committed rows of the sequence (its first token is
 * below seq_len) no less than it was; the committed rows are put under a scale
 * that grew.  Bytes of other rows stay as they are.
 *
 * DEVICE pointers but for batch and cache; asynchronous on `stream`.
 *   layer     of the cache, 0 .. n_layers - 1
 *   others    as for ooo_paged_append
 * Values that are not finite are stored as NaN and ask for no scale; values
 * beyond 448 * 2^119 become that.  A row without a place (ooo_paged_append)
 * gets its q and asks for no scale.  No two sequences' new rows may lie in one
 * block (a page that two tables name): its scale and rows would be of either.
 * Errors: as for ooo_paged_append; OOO_ERR_INVALID (layer).
 */
int ooo_paged_append8(const ooo_paged_batch* batch, const ooo_cache8* cache, int32_t layer, const void* qkv,
                      int64_t qkv_ld, const void* q_norm, const void* k_norm, float eps, const int32_t* depth,
                      double rope_theta, void* q_out, void* stream);

/*
 * ooo_paged_plan8 - as ooo_paged_plan, for ooo_paged_attn8 alone (a plan of
 * ooo_paged_plan gives NaN rows there, and the other way round).
 */
size_t ooo_paged_plan8_bytes(const ooo_paged_batch* batch);
int ooo_paged_plan8(const ooo_paged_batch* batch, void* plan, size_t plan_bytes, void* stream);

/*
 * ooo_paged_attn8 - as ooo_paged_attn, over one layer of an 8-bit cache: keys
 * and values are the numbers times their scales, exactly.
 */
size_t ooo_paged_attn8_workspace(const ooo_paged_batch* batch);
int ooo_paged_attn8(const ooo_paged_batch* batch, const ooo_cache8* cache, int32_t layer, const void* plan,
                    size_t plan_bytes, const void* q, float scale, void* out, void* workspace, size_t ws_bytes,
                    void* stream);

/*
 * ooo_paged_compact8 - as ooo_paged_compact, for every layer of the cache.  A
 * block that rows come into gets the largest scale of the blocks that these
 * come from, and where it holds committed rows no less than it had; its rows
 * are put under it (rounded to nearest even where they become subnormal).
 * Rows that are not moved by ooo_paged_compact ask for no scale.  No two
 * sequences' new rows may lie in one block (as for ooo_paged_append8).
 * Errors: as for ooo_paged_compact.
 */
int ooo_paged_compact8(const ooo_paged_batch* batch, const ooo_cache8* cache, const int32_t* path,
                       const int32_t* accept_len, int32_t path_cap, void* stream);

/*
 * ooo_paged_fork - sequences become continuations of others.  Sequence b with
 * a parent p = parent[b] gets the parent's length n = seq_len[p] and, in its
 * page table, the parent's entries of the n / page_rows full pages (both
 * sequences read those; nothing writes committed rows) and the page fresh[b]
 * behind them, into which the parent's n % page_rows committed rows of its open
 * page are copied, in all layers, K and V.  Other rows of the fresh page and
 * other entries of the table stay as they are.
 *
 * DEVICE pointers; asynchronous on `stream`.
 *   k_pages, v_pages   [n_layers] pools, layer_stride elements apart
 *   parent        [n_seqs] int32; below 0, or b itself: none
 *   fresh         [n_seqs] int32: a page that is in no table, for every
 *                 sequence with a parent
 *   seq_len_out, table_out   [n_seqs], [n_seqs][table_ld] int32: the batch's
 *                 own arrays (both), or others that do not overlap them (both).
 *                 In others every sequence is written, and a parent may itself
 *                 have a parent (all are read as they were: beams that change
 *                 places); in the batch's own, a child whose parent's entry
 *                 names another sequence is left as it is.
 * A sequence is left as it is, too, if its parent is no sequence or has a
 * length that is negative or fills its whole table, or if fresh[b] is no page,
 * or if the parent's open page holds rows and is none.  head_dim, dt and the
 * sizes come from the batch (row_start, anc_mask and the shared prompt are not
 * read).
 * Errors: as for ooo_paged_compact; OOO_ERR_INVALID (one of the outputs alone
 * is the batch's).
 *
 * ooo_paged_fork8 does the same for an 8-bit cache, with the scales of the
 * blocks that hold copied rows.
 */
int ooo_paged_fork(const ooo_paged_batch* batch, void* k_pages, void* v_pages, int32_t n_layers,
                   int64_t layer_stride, const int32_t* parent, const int32_t* fresh, int32_t* seq_len_out,
                   int32_t* table_out, void* stream);
int ooo_paged_fork8(const ooo_paged_batch* batch, const ooo_cache8* cache, const int32_t* parent,
                    const int32_t* fresh, int32_t* seq_len_out, int32_t* table_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* OOO_CACHE8_H */
