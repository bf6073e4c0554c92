// How a batch's attention is cut into pieces, shared by the plan's kernels,
// the attention kernels and the host.
//
// The query rows of a KV head are stacked: row i of a sequence gives G query
// rows i G .. i G + G - 1, one for each query head of the group.  A *block* is
// a set of query rows that read the same keys:
//   own blocks     up to `wide` consecutive query rows of one sequence (one
//                  block of up to `narrow` where there are few), against the
//                  sequence's own tokens;
//   shared blocks  up to `wide` query rows of the whole stack, against the
//                  shared prompt, which is so read once for many sequences.
// A block's keys go in tiles of 64, and its tiles are split evenly into
// *items*, one workgroup per KV head each, so that all items cost about the
// same: total cost / `target`.  An item leaves unnormalised sums and softmax
// statistics in *slots* of `group` query rows; a second kernel joins the slots
// of every row.  A block with one item and no shared part writes its output
// itself.
#pragma once

#include "paged.h"

namespace ooo {

constexpr int kTileKeys = 64;

struct PlanShape {
  int narrow, wide, group;         // query rows
  int cost_narrow, cost_wide;      // of a tile
  int target;                      // items of a KV head aimed at
  long long max_blocks, max_items, max_slots;
  long long off_blocks, off_seqs, off_items, off_rows, bytes;
};

// Item record (16 ints).
struct Item {
  int flags;   // kShared | kWide | kDirect
  int seq;
  int row0;    // the sequence's first row (0 for shared blocks)
  int q0, nq;  // query rows [q0, q0 + nq) of the sequence or of the stack
  int t0, t1;  // tiles
  int limit;   // keys of the block (those from limit on are not read)
  int len;     // own committed tokens (shared: the limit)
  int rows;    // the sequence's new rows
  int slot;    // first slot
  int pad[5];
};
static_assert(sizeof(Item) == 64, "item record");
enum { kShared = 1, kWide = 2, kDirect = 4 };

// Head of the plan.
struct PlanHead {
  int key[8];       // the sizes it was made for
  int items;
  int rows;         // new rows there are
  int shared_splits, shared_block, shared_slot0;
  int pad[3];
};
static_assert(sizeof(PlanHead) == 64, "plan head");

// Slots of one query row in its own part; the shared part follows from the
// head.  splits 0: the row is written by its item.
struct RowSlots {
  int slot, splits, stride, row;
};

inline PlanShape plan_shape(const ooo_paged_batch& b) {
  PlanShape s{};
  const bool bf = b.dt == OOO_BF16;
  s.group = bf ? 32 : 16;
  s.narrow = s.group;
  s.wide = bf ? 128 : 16;
  s.cost_narrow = s.cost_wide = 1;
  s.target = (bf ? 1 : 2) * device_cus() / b.n_kv_heads;
  if (s.target < 1) s.target = 1;
  const long long G = b.n_q_heads / b.n_kv_heads, q = b.n_rows * G;
  const long long stack = b.shared_len > 0 ? (q + s.group - 1) / s.group : 0;
  // a sequence's last block may be short, so one more than the full ones each
  s.max_blocks = b.n_seqs + q / s.wide;
  s.max_items = s.max_blocks + stack + s.target;
  s.max_slots = b.n_seqs + q / s.group + stack + (long long)(s.wide / s.group) * (s.target + (stack > 0));
  const auto up = [](long long n) { return (n + 63) / 64 * 64; };
  s.off_blocks = sizeof(PlanHead);
  s.off_seqs = up(s.off_blocks + s.max_blocks * 16);
  s.off_items = up(s.off_seqs + (b.n_seqs + 1) * 4ll);
  s.off_rows = s.off_items + s.max_items * (long long)sizeof(Item);
  s.bytes = s.off_rows + q * (long long)sizeof(RowSlots);
  return s;
}

// Whether the workgroups of the largest plan can be launched.
inline bool plan_grid_ok(const ooo_paged_batch& b, const PlanShape& s) {
  const double join = ((double)b.n_rows * (b.n_q_heads / b.n_kv_heads) / s.group + 1) * b.n_kv_heads * b.head_dim;
  return (double)s.max_items * b.n_kv_heads <= 1073741824.0 && join <= 1073741824.0;
}

// The sizes that a plan belongs to.
inline void plan_key(const ooo_paged_batch& b, int (&k)[8]) {
  k[0] = b.n_seqs;
  k[1] = b.n_rows;
  k[2] = b.n_q_heads;
  k[3] = b.n_kv_heads;
  k[4] = b.table_ld;
  k[5] = b.shared_len;
  k[6] = b.mask_words;
  k[7] = (b.page_rows << 12) + b.head_dim * 4 + (int)b.dt + 1;
}

}  // namespace ooo
