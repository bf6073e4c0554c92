// What the kernels over cache pages share: the batch descriptor as kernels
// take it, its checks, and the search for a row's sequence.
#pragma once

#include "device_common.h"
#include "ooo_batch.h"
#include "ooo_internal.h"

namespace ooo {

// ooo_paged_batch by value, with the page size as a shift.
struct Paged {
  const int32_t* row_start;
  const int32_t* seq_len;
  const int32_t* table;
  const int32_t* shared_pages;
  const uint64_t* mask;
  long long page_stride;
  int n_seqs, n_rows, table_ld, shared_len, page_shift, n_pages;
  int Hq, Hkv, G, W;
  int own_cap;  // tokens a page table holds
};

// Checks shared by every entry point; fills `p`.
inline int check_paged(const char* who, const ooo_paged_batch* b, Paged& p) {
  OOO_REQUIRE(b, OOO_ERR_INVALID, "%s: batch is null", who);
  OOO_REQUIRE(b->row_start && b->seq_len && b->page_table, OOO_ERR_INVALID,
              "%s: row_start, seq_len or page_table is null", who);
  OOO_REQUIRE(b->n_seqs >= 1 && b->n_rows >= 1 && b->table_ld >= 1 && b->n_pages >= 1, OOO_ERR_INVALID,
              "%s: n_seqs (%d), n_rows (%d), table_ld (%d) and n_pages (%d) must be >= 1", who, b->n_seqs, b->n_rows,
              b->table_ld, b->n_pages);
  OOO_REQUIRE(b->shared_len >= 0 && (b->shared_len == 0 || b->shared_pages), OOO_ERR_INVALID,
              "%s: shared_len is %d and shared_pages %s", who, b->shared_len, b->shared_pages ? "given" : "null");
  OOO_REQUIRE(b->n_q_heads >= 1 && b->n_kv_heads >= 1 && b->n_q_heads % b->n_kv_heads == 0, OOO_ERR_INVALID,
              "%s: n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", who, b->n_q_heads, b->n_kv_heads);
  OOO_REQUIRE(b->anc_mask ? b->mask_words >= 1 && b->mask_words <= 16 : b->mask_words == 0, OOO_ERR_INVALID,
              "%s: mask_words is %d (1 to 16 with anc_mask, 0 without)", who, b->mask_words);
  OOO_REQUIRE(b->dt == OOO_F32 || b->dt == OOO_BF16, OOO_ERR_INVALID, "%s: unknown dtype %d", who, (int)b->dt);
  OOO_REQUIRE(b->head_dim == 64 || b->head_dim == 128, OOO_ERR_UNSUPPORTED,
              "%s: head_dim %d not supported (64 or 128)", who, b->head_dim);
  OOO_REQUIRE(b->page_rows >= 16 && b->page_rows <= 65536 && (b->page_rows & (b->page_rows - 1)) == 0,
              OOO_ERR_UNSUPPORTED, "%s: page_rows %d not supported (a power of two, 16 to 65536)", who, b->page_rows);
  OOO_REQUIRE(b->n_seqs <= 65535, OOO_ERR_UNSUPPORTED, "%s: n_seqs %d above 65535", who, b->n_seqs);
  const int64_t own = (int64_t)b->table_ld * b->page_rows;
  OOO_REQUIRE(own <= (1 << 30) && b->shared_len <= (1 << 30), OOO_ERR_UNSUPPORTED,
              "%s: more than 2^30 tokens a sequence", who);
  OOO_REQUIRE((int64_t)b->n_rows * b->n_q_heads <= (1 << 28), OOO_ERR_UNSUPPORTED,
              "%s: n_rows * n_q_heads above 2^28", who);
  OOO_REQUIRE((int64_t)b->n_rows * b->mask_words <= (1 << 28), OOO_ERR_UNSUPPORTED,
              "%s: n_rows * mask_words above 2^28", who);  // kernels use 32-bit offsets into the mask
  const int64_t page = (int64_t)b->n_kv_heads * b->page_rows * b->head_dim;
  OOO_REQUIRE(b->page_stride >= page, OOO_ERR_INVALID, "%s: page_stride %lld below a page's %lld elements", who,
              (long long)b->page_stride, (long long)page);
  OOO_REQUIRE(page <= (1 << 30), OOO_ERR_UNSUPPORTED, "%s: a page of more than 2^30 elements", who);
  const int per16 = b->dt == OOO_BF16 ? 8 : 4;
  OOO_REQUIRE(b->page_stride % per16 == 0, OOO_ERR_UNSUPPORTED, "%s: page_stride is not a multiple of 16 bytes", who);
  p.row_start = b->row_start;
  p.seq_len = b->seq_len;
  p.table = b->page_table;
  p.shared_pages = b->shared_pages;
  p.mask = b->anc_mask;
  p.page_stride = b->page_stride;
  p.n_seqs = b->n_seqs;
  p.n_rows = b->n_rows;
  p.table_ld = b->table_ld;
  p.shared_len = b->shared_len;
  p.page_shift = __builtin_ctz((unsigned)b->page_rows);
  p.n_pages = b->n_pages;
  p.Hq = b->n_q_heads;
  p.Hkv = b->n_kv_heads;
  p.G = b->n_q_heads / b->n_kv_heads;
  p.W = b->mask_words;
  p.own_cap = (int)own;
  return OOO_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The new rows of all sequences that the buffers hold.
__device__ __forceinline__ int rows_of(const Paged& p) { return min(max(p.row_start[p.n_seqs], 0), p.n_rows); }
// A sequence's rows and own tokens, bounded to what buffers and tables hold
// (R: rows_of).
struct Seq {
  int row0, rows, len;
};
__device__ __forceinline__ Seq seq_of(const Paged& p, int b, int R) {
  Seq s;
  s.row0 = min(max(p.row_start[b], 0), R);
  s.rows = min(max(p.row_start[b + 1], s.row0), R) - s.row0;
  s.len = min(max(p.seq_len[b], 0), p.own_cap);
  return s;
}

// The sequence of row r (0 <= r < row_start[n]): the last b with
// row_start[b] <= r, where row_start rises from 0 (else any, to be checked
// against its rows), found by the whole wave, 64 bounds at a time: one round
// trip for 64 sequences, two for 4096.  Every lane gets the answer.
__device__ __forceinline__ int seq_of_row(const int32_t* row_start, int n, int r, int lane) {
  int lo = 0, len = n;  // the answer lies in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 63) / 64;
    const int at = lo + lane * step;
    const bool le = lane * step < len && row_start[at] <= r;
    const int k = max(__popcll(__ballot(le)), 1) - 1;
    lo += k * step;
    len = min(step, len - k * step);
  }
  return lo;
}

}  // namespace ooo
