// What the attention kernels over cache pages share: their arguments, the
// keys that a row sees and an item's pages.
#pragma once

#include "paged_plan.h"

namespace ooo {

struct PagedAttnArgs {
  Paged p;
  PlanHead want;        // key to compare with
  const uint8_t* plan;
  long long off_first_w, off_first_n, off_items_w, off_items_n, off_rows;
  int max_items_w, max_items_n, workers;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* part_o;        // [slot][Hkv] groups in fragment order
  float* part_ml;       // [slot][Hkv][group] (m, l)
  long long max_slots;
  float scale_log2e;    // bf16: its size
};

// Memory that no kernel writes while it is read here, the same address in the
// whole wave: scalar loads, which leave the count of vector loads (and so the
// waits for the LDS DMA) alone.
typedef const __attribute__((address_space(4))) int32_t* ScalarPtr;
__device__ __forceinline__ ScalarPtr scalar_ptr(const void* p) { return (ScalarPtr)(uintptr_t)p; }

// An item, in scalar registers (addresses of the LDS DMA follow from it).
__device__ __forceinline__ Item load_item(const uint8_t* items, int item) {
  const ScalarPtr src = scalar_ptr(items) + (size_t)item * (sizeof(Item) / 4);
  Item it{};
  int* dst = &it.flags;
#pragma unroll
  for (int k = 0; k < 11; ++k) dst[k] = src[k];
  return it;
}

// The plan's head, and whether the plan was made for these sizes.  All words
// are asked for at once, with the item's: tested one by one they were eight
// dependent loads ahead of everything else.
__device__ __forceinline__ PlanHead load_head(const PagedAttnArgs& a) {
  const ScalarPtr src = scalar_ptr(a.plan);
  PlanHead h{};
  int* dst = h.key;
#pragma unroll
  for (int k = 0; k < 16; ++k) dst[k] = src[k];
  return h;
}
// The wide items of one worker, in turn: f(item).
template <class F>
__device__ __forceinline__ void each_wide(const PagedAttnArgs& a, const PlanHead& h, int worker, F f) {
  bool first = true;
  const auto go = [&](int item) __attribute__((always_inline)) {
    if (!first) __syncthreads();  // the item before is joined
    first = false;
    f(item);
  };
  int item = worker < h.shared_workers ? worker : h.shared_items, step = h.shared_workers, end = h.shared_items;
  const int own = worker - h.own_first;
  bool more = own >= 0 && own < h.own_workers;
  while (true) {
    if (item >= end) {
      if (!more) break;
      const ScalarPtr fw = scalar_ptr(a.plan + a.off_first_w) + own;
      item = fw[0], end = min(fw[1], a.max_items_w), step = 1;
      more = false;
      continue;
    }
    go(item);
    item += step;
  }
}
__device__ __forceinline__ bool plan_fits(const PlanHead& h, const PlanHead& want) {
  int diff = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) diff |= h.key[k] ^ want.key[k];
  return diff == 0;
}

// Keys lo .. lo + 63 that the row sees, as bits.  len: own committed tokens;
// i: the row's index in its sequence; words: its mask words.
__device__ __forceinline__ uint64_t below(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t seen_in(const Paged& p, const Item& it, int i, const uint64_t* words, int lo) {
  if (it.flags & kShared) return below(it.limit - lo);
  if (!p.W) return below(min(it.limit, it.len + i + 1) - lo);
  const int off = lo - it.len;  // index among the new rows of key lo
  uint64_t w = off < 0 ? below(-off) : 0;
  if (off > -64) {
    const int x = off >> 6, sh = off & 63;  // floor division: x may be -1
    const uint64_t x0 = x >= 0 && x < p.W ? words[x] : 0, x1 = x + 1 < p.W ? words[x + 1] : 0;
    w |= sh ? (x0 >> sh) | (x1 << (64 - sh)) : x0;
  }
  return w & below(it.limit - lo);
}
__device__ __forceinline__ uint64_t seen(const Paged& p, const Item& it, int i, int row, int lo) {
  return seen_in(p, it, i, p.mask + (size_t)row * p.W, lo);
}
// First key that not every row of the block sees.
__device__ __forceinline__ int all_see(const Paged& p, const Item& it) {
  if (it.flags & kShared) return it.limit;
  return p.W ? it.len : min(it.limit, it.len + it.q0 / p.G + 1);
}

// Pages of one item: the page of key t (the same in the whole wave), page 0
// and `bad` where it is none.
struct Pages {
  ScalarPtr ids;
  int shift, n_pages;
  __device__ __forceinline__ Pages(const Paged& p, const Item& it)
      : ids(scalar_ptr(it.flags & kShared ? p.shared_pages : p.table + (size_t)it.seq * p.table_ld)),
        shift(p.page_shift),
        n_pages(p.n_pages) {}
  __device__ __forceinline__ int at(int t, bool& bad) const {
    const int id = ids[__builtin_amdgcn_readfirstlane(t >> shift)];
    const bool ok = id >= 0 && id < n_pages;
    bad = bad || !ok;
    return ok ? id : 0;
  }
};

}  // namespace ooo
