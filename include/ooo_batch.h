/*
 * ooo_batch.h - entry points of libooo for a batch of requests.
 *
 * A batch of requests that share one long prompt (tool schemas, system text)
 * and keep their own keys and values in cache pages (the step's counterparts
 * for many requests at once):
 *
 *   ooo_paged_append   q/k norms and rotation of a batch's new rows, q out,
 *                      k/v into the sequences' pages
 *   ooo_paged_plan     the split of a batch's attention work, once a step
 *   ooo_paged_attn     every new row attends to the shared prompt, its own
 *                      sequence's pages and its ancestors among the new rows
 *   ooo_paged_compact  moves the accepted rows of every sequence together
 *   ooo_sample         draws a token from each row's logits (temperature,
 *                      top-k, top-p, min-p; the random numbers are given)
 *
 * The conventions of ooo.h hold: status codes and ooo_last_error(), checks on
 * the host before anything is enqueued, asynchronous on `stream`, no device
 * memory allocated, no state between calls, deterministic results.
 */
#ifndef OOO_BATCH_H
#define OOO_BATCH_H

#include "ooo.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ooo_paged_batch - one batch of sequences over a pool of cache pages, as the
 * ooo_paged_* entry points read it.  The struct lives in HOST memory; the
 * arrays it points to are DEVICE memory and are read when the kernels run, so
 * one struct serves a captured step that is replayed while lengths and page
 * tables grow.
 *
 * A layer's pools k_pages, v_pages hold n_pages pages [n_kv_heads][page_rows]
 * [head_dim], page_stride elements apart.  The positions of a sequence b are
 *   0 .. shared_len - 1             the prompt that all sequences share: token
 *                                   t in page shared_pages[t / page_rows], row
 *                                   t % page_rows
 *   shared_len + 0 .. seq_len[b]-1  its own committed tokens: own token t in
 *                                   page page_table[b][t / page_rows]
 *   then its new rows               row i of the step is own token
 *                                   seq_len[b] + i
 * The new rows of all sequences lie behind each other: sequence b's are rows
 * row_start[b] .. row_start[b + 1] - 1 of q, qkv and out (none is allowed).
 * Rows from row_start[n_seqs] to n_rows are never touched.
 *
 *   n_seqs        sequences (1 .. 65535)
 *   n_rows        rows the step's buffers hold; row_start[n_seqs] <= n_rows;
 *                 n_rows * n_q_heads and n_rows * mask_words up to 2^28
 *   row_start     [n_seqs + 1] int32, non-decreasing, row_start[0] == 0
 *                 (rows ahead of row_start[0] would be no sequence's)
 *   seq_len       [n_seqs] int32, >= 0
 *   page_table    [n_seqs][table_ld] int32
 *   shared_pages  [ceil(shared_len / page_rows)] int32 (NULL if shared_len is 0)
 *   page_rows     a power of two from 16 to 65536
 *   page_stride   elements from one page to the next, a multiple of 8
 *                 (bf16) or 4 (float32) and at least n_kv_heads * page_rows *
 *                 head_dim
 *   anc_mask      NULL: a sequence's new rows are a chain, row i sees the new
 *                 rows 0 .. i.  Or [n_rows][mask_words] uint64 (mask_words 1
 *                 to 16, 0 with NULL): row i of a sequence sees its new row j
 *                 where bit j is set (a trie's ancestors, ooo_pack_tree);
 *                 new rows from 64 * mask_words on are seen by none
 *   dt            OOO_BF16 or OOO_F32: q, qkv, norms, out and pages
 * head_dim 64 or 128; query head h reads KV head h / (n_q_heads / n_kv_heads).
 *
 * What the host cannot check is bounded on the device: rows and tokens past
 * n_rows or past table_ld * page_rows are left out, and a page outside
 * [0, n_pages) is never dereferenced (each entry point says what comes then).
 * Where row_start falls, attention gives NaN rows and the others leave out the
 * rows that lie outside their sequence's range.
 */
typedef struct {
  int32_t n_seqs;
  int32_t n_rows;
  const int32_t* row_start;
  const int32_t* seq_len;
  const int32_t* page_table;
  const int32_t* shared_pages;
  const uint64_t* anc_mask;
  int64_t page_stride;
  int32_t table_ld;
  int32_t shared_len;
  int32_t page_rows;
  int32_t n_pages;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t mask_words;
  ooo_dtype dt;
} ooo_paged_batch;

/*
 * ooo_paged_append - the batch's counterpart of ooo_qk_norm_rope: per-head
 * RMSNorm of q and k, rotate-half rotation at the row's position, q to q_out
 * and k, v to the row's own place in the pages.
 *
 * DEVICE pointers; asynchronous on `stream`.
 *   qkv       [n_rows][(n_q_heads + 2 n_kv_heads) head_dim], q heads, then k
 *             heads, then v heads; rows qkv_ld elements apart (a multiple of
 *             16 bytes)
 *   q_norm, k_norm   [head_dim], or NULL (no norm)
 *   depth     NULL: row i of a sequence stands at shared_len + seq_len + i; or
 *             [n_rows] int32: at shared_len + seq_len + depth[row]
 *   q_out     [n_rows][n_q_heads][head_dim]; must not alias qkv
 *   k_pages, v_pages   one layer's pools, written at the new rows only
 * A row whose place lies past its page table or in a page outside
 * [0, n_pages) gets its q but no place in the pages.  Two rows in one place
 * (a page that two sequences' tables name) leave either's value.
 * Errors: OOO_ERR_INVALID (null pointers, sizes out of the ranges above,
 * eps < 0, rope_theta <= 0), OOO_ERR_UNSUPPORTED (head_dim, page_rows,
 * strides or pointers not a multiple of 16 bytes), OOO_ERR_HIP.
 */
int ooo_paged_append(const ooo_paged_batch* batch, const void* qkv, int64_t qkv_ld, const void* q_norm,
                     const void* k_norm, float eps, const int32_t* depth, double rope_theta, void* q_out,
                     void* k_pages, void* v_pages, void* stream);

/*
 * ooo_paged_plan - how the batch's attention is cut into pieces of equal
 * work, from row_start and seq_len (read on the device; no host
 * synchronisation).  One plan serves every layer of the step; it is made anew
 * when row_start, seq_len, shared_len or the sizes change.
 *   plan, plan_bytes   device memory (16-byte aligned) of ooo_paged_plan_bytes(batch)
 *                      bytes, which depend on n_seqs, n_rows, table_ld,
 *                      page_rows, shared_len, heads, head_dim and dt alone
 *                      and not on what the device arrays hold
 * Errors: as for ooo_paged_append; OOO_ERR_CAPACITY (plan_bytes).  The size
 * queries return 0 for a batch that is refused.
 */
size_t ooo_paged_plan_bytes(const ooo_paged_batch* batch);
int ooo_paged_plan(const ooo_paged_batch* batch, void* plan, size_t plan_bytes, void* stream);

/*
 * ooo_paged_attn - one layer of attention for the batch: row i of sequence b
 * attends to the shared prompt, to the sequence's own committed tokens and to
 * the new rows it sees (itself among them; their k and v are in the pages,
 * ooo_paged_append).  The shared prompt is read once for all sequences: their
 * rows are stacked against it, and the parts are joined by their softmax
 * statistics (float32).
 *
 * DEVICE pointers; asynchronous on `stream`.
 *   plan      of ooo_paged_plan for this batch.  A plan that was made for
 *             other sizes gives NaN rows; lengths come from the plan
 *   q         [n_rows][n_q_heads][head_dim] (16-byte aligned, as the pools and out)
 *   scale     score scale, normally 1/sqrt(head_dim); any finite one (times
 *             log2(e) too): 0 weighs all seen keys alike
 *   out       [n_rows][n_q_heads][head_dim], the type of q; must not alias
 *   workspace, ws_bytes   ooo_paged_attn_workspace(batch) bytes (16-byte
 *             aligned; on the same sizes as ooo_paged_plan_bytes)
 * A row that sees no key at all is zero.  A key that a row does not see has
 * no influence on it, whatever its k and v hold (NaN and infinities too).  A
 * page outside [0, n_pages) where keys are read gives NaN rows to those who
 * read it (a shared page: to all), and to rows of the same sequence that are
 * worked on together with them (up to 128 query rows of a KV head) though they
 * do not see its keys.
 * Errors: as for ooo_paged_append; OOO_ERR_INVALID (a scale that is not finite),
 * OOO_ERR_CAPACITY (ws_bytes, plan_bytes).
 */
size_t ooo_paged_attn_workspace(const ooo_paged_batch* batch);
int ooo_paged_attn(const ooo_paged_batch* batch, const void* plan, size_t plan_bytes, const void* q,
                   const void* k_pages, const void* v_pages, float scale, void* out, void* workspace,
                   size_t ws_bytes, void* stream);

/*
 * ooo_paged_compact - commit the accepted rows of every sequence: the batch's
 * counterpart of ooo_kv_compact.  For every layer, KV head, K and V: own
 * token seq_len[b] + path[b][d] moves to own token seq_len[b] + d, for d = 0 ..
 * accept_len[b].  (The caller then adds accept_len[b] + 1 to seq_len[b].)
 *
 * DEVICE pointers; asynchronous on `stream`.
 *   k_pages, v_pages   [n_layers] pools, layer_stride elements apart, updated
 *                 in place
 *   path          [n_seqs][path_cap] int32, each a root path of the sequence's
 *                 trie (strictly increasing, as ooo_accept writes it)
 *   accept_len    [n_seqs] int32; -1, or a length that path_cap does not
 *                 hold, moves no row of that sequence
 * Entries of path outside the sequence's new rows, and rows whose place is
 * past the page table or in a page outside [0, n_pages), are not moved.  No
 * two sequences' new rows may lie in one place (as for ooo_paged_append).
 * Errors: as for ooo_paged_append; OOO_ERR_INVALID (n_layers or path_cap < 1).
 */
int ooo_paged_compact(const ooo_paged_batch* batch, void* k_pages, void* v_pages, int32_t n_layers,
                      int64_t layer_stride, const int32_t* path, const int32_t* accept_len, int32_t path_cap,
                      void* stream);

/*
 * ooo_sample - one token from each row of logits, with the row's own settings
 * and a given random number.
 *
 * DEVICE pointers; asynchronous on `stream`.
 *   logits       [n_rows][vocab] float32 (ooo_lmhead_argmax writes them) or
 *                bf16, rows ld >= vocab elements apart (any alignment of the
 *                type)
 *   temperature  [n_rows] float32, or NULL (1): T; not above 0: the row's
 *                largest logit, whatever the other settings
 *   top_k        [n_rows] int32, or NULL: keep the k likeliest (below 1: all)
 *   top_p        [n_rows] float32, or NULL: of those, keep the fewest likeliest
 *                whose probabilities reach top_p of theirs (1 or more: all)
 *   min_p        [n_rows] float32, or NULL: keep those at least min_p as
 *                likely as the likeliest (0 or less: all)
 *   u            [n_rows] float32 in [0, 1)
 *   ids          [n_rows] int32: with the row's tokens in the order of their
 *                logits (the largest first, equal ones by index) and weights
 *                w = exp((x - max) / T), the first kept token at which the
 *                running sum of the weights exceeds u times the kept total
 *   prob         NULL, or [n_rows] float32: its weight over the kept total
 *   kept         NULL, or [n_rows] int32: how many tokens were kept (>= 1)
 * All three filters keep a head of that order; the shortest counts, and the
 * likeliest token is always kept.  Logits of -inf and NaN are never drawn or
 * counted; a row of nothing else gives id -1, prob 0, kept 0.  Logits of +inf
 * share the whole weight.  Weights are sums of 64-bit whole numbers (2^-42 of
 * the largest or finer), so results do not depend on any order of addition.
 *   workspace, ws_bytes   ooo_sample_workspace(n_rows, vocab) bytes (16-byte aligned)
 * Errors: OOO_ERR_INVALID (null pointers, sizes < 1, ld < vocab, unknown
 * dtype), OOO_ERR_UNSUPPORTED (vocab above 2^20, n_rows above 65535, workspace
 * not aligned), OOO_ERR_CAPACITY, OOO_ERR_HIP.
 */
size_t ooo_sample_workspace(int32_t n_rows, int32_t vocab);
int ooo_sample(const void* logits, int64_t ld, ooo_dtype dt, int32_t n_rows, int32_t vocab,
               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
               const float* u, int32_t* ids, float* prob, int32_t* kept, void* workspace, size_t ws_bytes,
               void* stream);

#ifdef __cplusplus
}
#endif

#endif /* OOO_BATCH_H */
