// The order of a wide attention item's copies (paged_attn_bf16.h, paged_attn8.h):
// what its barriers wait for and which of its tiles go through the loop's body
// without conditions.  For the kernels and for a host's model of them.
//
// A wave asks for its share of K and V of the item's tiles, and its copies land in
// the order in which it asked.  Barrier m promises K of tile m and V of tile m - 1;
// ahead of it a wave has asked for K up to tile m + 2 and V up to tile m, these two
// last, in either order.
#pragma once

namespace ooo {

// Copies of a wave that barrier m of an item leaves on their way.
__host__ __device__ __forceinline__ constexpr int copies_left(int m, int tiles) {
  return m + 2 < tiles ? 2 : m < tiles ? 1 : 0;
}

// Where a run of tiles without conditions, from tile n on, ends.  seen: tiles of
// which every row sees every key; full: tiles whose keys all exist; window: the
// first tile whose address is not at hand.  Its body copies K of tile n + 5 and V
// of n + 2 or n + 3 without asking whether there are any (where there is none, the
// last tile's again), so it ends five before a tile that is not full or has no
// address yet.  And its barrier n + 2 always leaves two copies on their way, K of
// tile n + 4 and V of n + 2.  Where the careful body ahead of the run had no K of
// tile n + 4 to copy, it leaves the one before these: of an item with one tile none
// that matters, with four K of tile 3, but with two and three V of tile 1, which the
// barrier promises; such items have no run.  (Later runs of longer items begin
// behind a copy of K of tile n + 4.)
__host__ __device__ __forceinline__ int plain_end(int tiles, int seen, int full, int window) {
  if (tiles == 2 || tiles == 3) return 0;
  const int care = full < window ? full : window, end = seen < tiles ? seen : tiles;
  return care < tiles && care - 5 < end ? care - 5 : end;
}

}  // namespace ooo
