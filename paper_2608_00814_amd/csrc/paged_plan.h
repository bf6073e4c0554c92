// How a batch's attention is cut into pieces, shared by the plan's kernels,
// the attention kernels and the host.
//
// The query rows of a KV head are stacked: row i of a sequence gives G query
// rows i G .. i G + G - 1, one for each query head of the group.  A *block* is
// a set of query rows that read the same keys:
//   own blocks     up to `wide` consecutive query rows of one sequence, or up
//                  to `narrow` where its rows are no more or its keys few,
//                  against the sequence's own tokens;
//   shared blocks  the same of the whole stack, against the shared prompt,
//                  which is so read once for many sequences.
// A KV head's work goes to `workers` workgroups, all on the chip at once:
//  * the first ones take the wide shared blocks, each cut into the same number
//    of runs of its tiles of 64 keys.  A run of a block is an *item*; the items
//    are dealt out with the block index moving fastest, so that workgroups
//    that run at the same time read the same part of the prompt and share it
//    in their XCD's L2.  (Cut into equal runs one block behind the other, the
//    balance is perfect, but each workgroup is in another place of the prompt:
//    eight tries of 64 over a 4k prompt took 69 us so, 53 dealt out like this.)
//  * the next take the sequences' own wide blocks, one behind the other, in
//    runs of equal cost: a block's tiles and, ahead of them, as many as the
//    start and end of an item cost (runs of equal length left four prompts of
//    300 to 512 rows with workgroups 13 us behind the others);
//  * the last take the narrow blocks' half-tiles of 32 keys in the same way, a
//    run for each of their waves.
// The numbers of workgroups and runs are those that finish first by the costs
// of their kernels (PlanCosts).  The part of a block in one run leaves unnormalised sums and softmax
// statistics in *slots* of `group` query rows, and a second kernel joins the
// slots of every row.  A block of one item and without a shared part writes
// its output itself.
#pragma once

#include "paged.h"

namespace ooo {

constexpr int kTileKeys = 64;
// Up to so many tiles of keys, 128 query rows are cheaper as four narrow blocks,
// one wave's work each and eight at a time on a worker, than as a wide one,
// whose start and end take longer than its tiles (38 tries of 46 rows with no
// prompt to speak of: 60 us in wide blocks, 46 so; 8 tiles are no better).
constexpr int kShortTiles = 4;
constexpr int kSplitMost = 4;  // extra items of the shared blocks: at most so many times the workers

// Waves of a float32 worker, and workers on a CU at once (the kernel keeps 148
// registers at head_dim 64 and 249 at 128; at 128 forced to 168, it spills and
// takes twice the time, and eight waves a worker, one of which fills a CU, take
// 10% longer).
constexpr int kF32Waves = 4;
__host__ __device__ constexpr int f32_per_cu(int head_dim) { return head_dim == 64 ? 3 : 2; }

struct PlanShape {
  int narrow, wide, group;  // query rows (narrow 0: there are no narrow blocks)
  int waves;                // of a worker, where narrow blocks are one wave's work
  int workers;              // workgroups of a KV head
  long long max_blocks, max_items_w, max_items_n, max_slots;
  long long off_blocks, off_seqs, off_first_w, off_first_n, off_items_w, off_items_n, off_rows, bytes;
};

// Costs in 100 cycles at head_dim 128 (half of them at 64), as measured: a wide
// tile of a worker; an item's start (its record, pages, queries and first
// tiles, one behind the other) and end; a half-tile of a narrow worker, whose
// eight waves have 128 KiB on their way; and a half-tile at the chip's share of
// the HBM rate.
struct PlanCosts {
  float tile, item, half, half_hbm;
};

// Item record (16 ints).
struct Item {
  int flags;   // kShared | kDirect
  int seq;
  int row0;    // the sequence's first row (0 for shared blocks)
  int q0, nq;  // query rows [q0, q0 + nq) of the sequence or of the stack
  int t0, t1;  // tiles (wide) or half-tiles (narrow)
  int limit;   // keys of the block (those from limit on are not read)
  int len;     // own committed tokens (shared: the limit)
  int rows;    // the sequence's new rows
  int slot;    // first slot
  int pad[5];
};
static_assert(sizeof(Item) == 64, "item record");
enum { kShared = 1, kDirect = 4 };

// Head of the plan.
struct PlanHead {
  int key[8];       // the sizes it was made for
  int rows;         // new rows there are
  int shared_block; // query rows of a shared block (0: no shared part)
  int shared_items, shared_workers;              // wide ones
  int own_first, own_workers;                    // workers with own wide runs
  int narrow_first, narrow_workers;
};
static_assert(sizeof(PlanHead) == 64, "plan head");

// Slots of one block: `splits` times `groups` of them, from `slot` on.
// splits 0: written by its item.
struct BlockSlots {
  int slot, splits, groups, pad;
};
// Slots of one query row: in the shared part and in its own.
struct RowSlots {
  struct Part {
    int slot, splits, stride, row;  // splits 0: none, or written by its item
  } part[2];
};

inline PlanShape plan_shape(const ooo_paged_batch& b) {
  PlanShape s{};
  const bool bf = b.dt == OOO_BF16;
  s.group = bf ? 32 : 16;
  s.narrow = bf ? 32 : 0;
  s.wide = bf ? 128 : 16;
  s.waves = bf ? 8 : 0;
  s.workers = (bf ? 1 : f32_per_cu(b.head_dim)) * device_cus() / b.n_kv_heads;
  if (s.workers < 1) s.workers = 1;
  const long long G = b.n_q_heads / b.n_kv_heads, q = b.n_rows * G;
  const long long shared = b.shared_len > 0 ? (q + s.wide - 1) / s.wide : 0;
  const long long own = b.n_seqs + q / s.wide;  // a sequence's last block may be short
  const long long narrow = bf ? b.n_seqs + q / s.narrow + (b.shared_len > 0 ? q / s.narrow + 1 : 0) : 0;
  s.max_blocks = shared + own + narrow;
  s.max_items_w = shared + own + (kSplitMost + 1ll) * s.workers;
  s.max_items_n = bf ? narrow + (long long)s.waves * s.workers : 0;
  const long long per_wide = s.wide / s.group, runs = s.workers * (per_wide + s.waves);
  s.max_slots = b.n_seqs + 1 + q / s.group + (shared + (long long)kSplitMost * s.workers) * per_wide + runs;
  const auto up = [](long long n) { return (n + 63) / 64 * 64; };
  s.off_blocks = sizeof(PlanHead);
  s.off_seqs = up(s.off_blocks + s.max_blocks * (long long)sizeof(BlockSlots));
  s.off_first_w = up(s.off_seqs + (b.n_seqs + 1) * 4ll);
  s.off_first_n = up(s.off_first_w + (s.workers + 1) * 4ll);
  s.off_items_w = up(s.off_first_n + (s.waves * s.workers + 1) * 4ll);
  s.off_items_n = s.off_items_w + s.max_items_w * (long long)sizeof(Item);
  s.off_rows = s.off_items_n + s.max_items_n * (long long)sizeof(Item);
  s.bytes = s.off_rows + q * (long long)sizeof(RowSlots);
  return s;
}

// Whether the workgroups of the largest plan can be launched.
inline bool plan_grid_ok(const ooo_paged_batch& b, const PlanShape& s) {
  const double join = ((double)b.n_rows * (b.n_q_heads / b.n_kv_heads) / s.group + 1) * b.n_kv_heads * b.head_dim;
  return (double)s.workers * b.n_kv_heads <= 1073741824.0 && join <= 1073741824.0;
}

// The sizes that a plan belongs to (eight: and pages of 8-bit numbers).
inline void plan_key(const ooo_paged_batch& b, bool eight, int (&k)[8]) {
  k[0] = b.n_seqs;
  k[1] = b.n_rows;
  k[2] = b.n_q_heads;
  k[3] = b.n_kv_heads;
  k[4] = b.table_ld;
  k[5] = b.shared_len;
  k[6] = b.mask_words;
  k[7] = (b.page_rows << 12) + b.head_dim * 4 + (int)b.dt + 1 + (eight ? 2 : 0);
}

}  // namespace ooo
