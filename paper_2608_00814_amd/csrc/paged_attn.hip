// Attention of a batch over a shared prompt and each sequence's own cache
// pages.  paged_plan.h says how the work is cut; here are the plan's kernels,
// the attention over one item and the join of the items' parts.
//
// For a query row, softmax(s q K^T) V over any split of its keys is joined
// from the parts' row maxima m, sums l = sum exp2(x - m) and unnormalised
// outputs O: O = sum_s exp2(m_s - m) O_s / sum_s exp2(m_s - m) l_s.  That is
// what lets the shared prompt be read once, for the stacked rows of all
// sequences, and long sequences be split.  Parts and statistics are float32.
#include "paged_attn8.h"
#include "paged_attn_bf16.h"

namespace ooo {
namespace {

constexpr int kPlanThreads = 512;

// ------------------------------------------------------------------- plan
// Whether query rows against so many keys go to wide blocks.
__device__ __forceinline__ bool wide_rows(const PlanShape& s, int rows, int keys) {
  return rows > s.narrow && (s.narrow == 0 || keys > kShortTiles * kTileKeys);
}
__device__ __forceinline__ int keys_of(const Paged& p, const Seq& q) {
  return min(q.len + (p.W ? min(q.rows, 64 * p.W) : q.rows), p.own_cap);
}

// What a thread of the plan looks at: one shared block, or one sequence.
struct Entry {
  Seq q;
  int rows;     // query rows of all its blocks
  int block;    // query rows of a block
  int n;        // blocks
  bool shared, wide;
  // block j: its query rows, the keys they can see and its length, in tiles
  // (wide) or half-tiles
  __device__ __forceinline__ void at(const Paged& p, int j, int& nq, int& limit, int& len) const {
    nq = min(block, rows - j * block);
    if (shared) {
      limit = p.shared_len;
    } else {
      const int last = (j * block + nq - 1) / p.G;
      limit = min(q.len + (p.W ? min(q.rows, 64 * p.W) : last + 1), p.own_cap);
    }
    len = wide ? (limit + kTileKeys - 1) / kTileKeys : (limit + kTileKeys / 2 - 1) / (kTileKeys / 2);
  }
};
__device__ __forceinline__ Entry entry_of(const Paged& p, const PlanShape& s, int e, int shared, int sblock, int R) {
  Entry x;
  const int stack = R * p.G;
  x.shared = e < shared;
  x.q = x.shared ? Seq{0, 0, 0} : seq_of(p, e - shared, R);
  x.rows = x.shared ? min(sblock, stack - e * sblock) : x.q.rows * p.G;
  x.wide = x.shared ? sblock > s.narrow : wide_rows(s, x.rows, keys_of(p, x.q));
  x.block = x.wide ? s.wide : s.narrow;
  x.n = x.rows > 0 ? (x.rows + x.block - 1) / x.block : 0;
  return x;
}

// Exclusive scan of N counts over the workgroup; the totals go to every thread.
template <int N>
__device__ __forceinline__ void scan(long long (&v)[N], long long (&total)[N]) {
  __shared__ long long sh[N][kPlanThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const long long own = v[n];
    for (int off = 1; off < 64; off <<= 1) {
      const long long x = __shfl_up(v[n], off, 64);
      if (lane >= off) v[n] += x;
    }
    if (lane == 63) sh[n][wave] = v[n];
    v[n] -= own;
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    total[n] = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      if (w < wave) v[n] += sh[n][w];
      total[n] += sh[n][w];
    }
  }
}

// How the workers of a KV head are shared out.
struct Deal {
  int splits, shared_workers, own_workers, narrow_workers;
};
constexpr PlanCosts kCosts{21.f, 160.f, 5.f, 0.05f};
// 8-bit pages: half the bytes of a half-tile, and wide tiles that convert.  256
// rows over 32k with up to 4k own take 306 us at halves of 3.5 to 4 and shares of
// HBM of 0.015 to 0.04, and 346 at 2.5, 325 at 4.5 to 7, 328 at a share of 0.05,
// 690 at a half of 0.5; own keys alone 206 from 0.025 on and 236 at 0.015.  Of
// fifteen shapes (32 to 300 rows over up to 32k and 16k own, tries, prompts, heads of
// 64) these take within 2% of the best of tiles of 21 to 31, halves of 3 to 4.5 and
// shares of 0.025 to 0.045, but for 64 rows of 40 heads over 12k (50 us; 46 at a tile
// of 21) and 128 rows over 16k with 4k own (122; 118 at 0.045); a share of 0.025 or
// 0.045 or a tile of 21 costs 100 rows over 20k with 8k own 11 to 14%, a tile of 31
// the 256 rows 13%, a half of 4.5 the same at heads of 64 9%; halves of 3 nothing.
constexpr PlanCosts kCosts8{26.f, 160.f, 3.5f, 0.033f};

// The deal that finishes first, for every lane of a wave, each of which tries
// its share of the split counts (one lane alone took 40 us for 65 of them).
// blocks, tiles: of the wide shared part; own: tiles of the sequences' wide
// blocks; halves: of the narrow blocks.
__device__ Deal deal_workers(const Paged& p, const PlanShape& s, const PlanCosts& cost, int blocks, int tiles,
                             long long own, long long halves, bool half_dim, int lane) {
  const int W = s.workers;
  const float tile = half_dim ? 0.5f * cost.tile : cost.tile, half = half_dim ? 0.5f * cost.half : cost.half;
  const float hbm = (half_dim ? 0.5f : 1.f) * cost.half_hbm * p.Hkv * (float)halves;
  Deal best{1, 0, 0, 0};
  float least = INFINITY;
  const int kinds = (blocks > 0) + (own > 0) + (halves > 0);
  const float co = (float)own * tile, cn = (float)halves * half;
  if (W <= kinds) {  // every worker takes a share of everything
    int n = blocks > 0 ? (W + blocks - 1) / blocks : 1;
    return Deal{max(min(n, tiles), 1), W, W, W};
  }
  const int room = W - (own > 0) - (halves > 0);
  const int most = blocks > 0 ? min(max(tiles, 1), kSplitMost * W / blocks + 1) : 1;
  for (int n = lane + 1; n <= most; n += 64) {
    const int items = blocks * n, k0 = max((items + room - 1) / room, 1);
    for (int k = k0; k <= k0 + 2; ++k) {
      const int ws = (items + k - 1) / k, rest = W - ws;
      int wo = own > 0 ? rest : 0, wn = halves > 0 ? rest : 0;
      if (own > 0 && halves > 0) {
        wo = (int)(rest * (co / (co + cn)) + 0.5f);
        wo = min(max(wo, 1), rest - 1);
        wn = rest - wo;
      }
      float t = blocks > 0 ? k * ((float)((tiles + n - 1) / n) * tile + cost.item) : 0.f;
      if (wo > 0) t = fmaxf(t, co / wo + cost.item);
      if (wn > 0) t = fmaxf(t, fmaxf(cn / wn, hbm));
      if (t < least) least = t, best = Deal{n, ws, wo, wn};
    }
  }
  for (int off = 32; off > 0; off /= 2) {  // of equal ones the one of fewer splits
    const float t = __shfl_xor(least, off, 64);
    const Deal d{__shfl_xor(best.splits, off, 64), __shfl_xor(best.shared_workers, off, 64),
                 __shfl_xor(best.own_workers, off, 64), __shfl_xor(best.narrow_workers, off, 64)};
    if (t < least || (t == least && d.splits < best.splits)) least = t, best = d;
  }
  return best;
}

// One workgroup, once a step.  First the lengths, from them the deal, then the
// items and slots of every entry behind those of the entries before it.  A
// sequence is one thread's work, block by block, so the time grows with the
// blocks of the longest one, 1.4 us each.  With plan_rows_kernel (4 to 6 us): 16
// us for 64 sequences of a row, 18 for 256, 75 for 4096; 19 for 8 of 64 rows of
// four query heads a group, 59 for one of 1024, 190 for one of 4096 and 695 for
// one of 16384 (128 wide blocks in 4096 rows); in float32, whose blocks are an
// eighth of that, 36 for 3 of 25 rows, 190 for one of 512, 1370 for one of 4096.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(Paged p, PlanShape s, PlanCosts cost, PlanHead head,
                                                            int half_dim, uint8_t* plan) {
  BlockSlots* const blocks = reinterpret_cast<BlockSlots*>(plan + s.off_blocks);
  int* const seq_block = reinterpret_cast<int*>(plan + s.off_seqs);
  int* const first_w = reinterpret_cast<int*>(plan + s.off_first_w);
  int* const first_n = reinterpret_cast<int*>(plan + s.off_first_n);
  Item* const items_w = reinterpret_cast<Item*>(plan + s.off_items_w);
  Item* const items_n = reinterpret_cast<Item*>(plan + s.off_items_n);
  const int tid = threadIdx.x;
  const int R = rows_of(p);
  const int stack = R * p.G;  // query rows of a KV head
  const bool swide = wide_rows(s, stack, p.shared_len);
  const int sblock = swide ? s.wide : s.narrow;
  const int sblocks = p.shared_len > 0 && stack > 0 ? (stack + sblock - 1) / sblock : 0;
  // entries: a narrow shared block, then the sequences
  const int lead = swide ? 0 : sblocks, entries = lead + p.n_seqs;
  const int tiles = (p.shared_len + kTileKeys - 1) / kTileKeys, per_wide = s.wide / s.group;
  // what an item's start and end cost, in wide tiles and in half-tiles of a wave
  const int lead_w = half_dim ? 16 : 8, lead_n = half_dim ? 6 : 3;
  __shared__ Deal deal_s;
  __shared__ int falls_s;
  if (tid == 0) falls_s = 0;
  bool falls = false;

  long long all[3] = {0, 0, swide ? sblocks : 0};  // own wide tiles, narrow half-tiles, blocks
  for (int e0 = 0; e0 < entries; e0 += kPlanThreads) {
    long long v[3] = {0, 0, 0}, t[3];
    const int e = e0 + tid;
    if (e < entries) {
      const Entry x = entry_of(p, s, e, lead, sblock, R);
      v[2] = x.n;
      falls |= !x.shared && p.row_start[e - lead + 1] < p.row_start[e - lead];
      for (int j = 0; j < x.n; ++j) {
        int nq, limit, len;
        x.at(p, j, nq, limit, len);
        v[x.wide ? 0 : 1] += len + (x.wide ? lead_w : lead_n);
      }
    }
    scan<3>(v, t);
    if (e >= lead && e < entries) seq_block[e - lead] = (int)min(all[2] + v[2], s.max_blocks);
#pragma unroll
    for (int k = 0; k < 3; ++k) all[k] += t[k];
  }
  if (falls) falls_s = 1;
  const int wblocks = swide ? sblocks : 0;
  if (tid < 64) {
    const Deal d = deal_workers(p, s, cost, wblocks, tiles, all[0], all[1], half_dim != 0, tid);
    if (tid == 0) deal_s = d;
  }
  __syncthreads();
  // Sequences overlap where row_start falls, and their blocks, items and slots
  // are more than there is room for, without bound.  Such a plan has no work and
  // a key that fits no batch.
  if (falls_s) {
    head.key[0] = 0;
    if (tid == 0) *reinterpret_cast<PlanHead*>(plan) = head;
    return;
  }
  const Deal d = deal_s;
  const int runs_w = max(d.own_workers, 1), runs_n = max(d.narrow_workers, 1) * max(s.waves, 1);
  const long long len_w = max((all[0] + runs_w - 1) / runs_w, 1ll), len_n = max((all[1] + runs_n - 1) / runs_n, 1ll);

  // the wide shared blocks' items, and their slots block by block
  const int per = (tiles + d.splits - 1) / d.splits, splits = wblocks ? (tiles + per - 1) / per : 0;
  const int shared_items = wblocks * splits;
  for (int k = tid; k < shared_items; k += kPlanThreads) {
    const int sp = k / wblocks, b = k - sp * wblocks;
    Item it{};
    it.flags = kShared;
    it.q0 = b * sblock;
    it.nq = min(sblock, stack - it.q0);
    it.t0 = sp * per;
    it.t1 = min(it.t0 + per, tiles);
    it.limit = it.len = p.shared_len;
    it.slot = (b * splits + sp) * per_wide;
    if (k < s.max_items_w) items_w[k] = it;
    if (sp == 0 && b < s.max_blocks) blocks[b] = BlockSlots{it.slot, splits, per_wide, 0};
  }

  // wide and narrow position, wide and narrow items, slots
  long long at[5] = {0, 0, shared_items, 0, (long long)shared_items * per_wide};
  long long blk = wblocks;
  for (int e0 = 0; e0 < entries; e0 += kPlanThreads) {
    const int e = e0 + tid;
    Entry x{};
    long long pos[3] = {0, 0, 0}, tp[3];
    if (e < entries) {
      x = entry_of(p, s, e, lead, sblock, R);
      pos[2] = x.n;
      for (int j = 0; j < x.n; ++j) {
        int nq, limit, len;
        x.at(p, j, nq, limit, len);
        pos[x.wide ? 0 : 1] += len + (x.wide ? lead_w : lead_n);
      }
    }
    scan<3>(pos, tp);
    const long long run = x.wide ? len_w : len_n;
    const int ahead = x.wide ? lead_w : lead_n;
    // items of a block from position q on: one for each run that it has a part
    // in, but none for a run that ends in its first `ahead` positions
    const auto pieces = [&](long long q, int len) {
      const int k = (int)((q + ahead + len - 1) / run - q / run) + 1;
      const long long in_lead = (q + ahead) / run - q / run;  // runs that end there
      return k - (int)in_lead;
    };
    long long p0 = x.wide ? at[0] + pos[0] : at[1] + pos[1];
    long long n[3] = {0, 0, 0}, tn[3];  // wide items, narrow items, slots
    {
      long long q = p0;
      for (int j = 0; j < x.n; ++j) {
        int nq, limit, len;
        x.at(p, j, nq, limit, len);
        const int k = pieces(q, len);
        n[x.wide ? 0 : 1] += k;
        if (sblocks || k > 1) n[2] += (long long)k * ((nq + s.group - 1) / s.group);
        q += ahead + len;
      }
    }
    scan<3>(n, tn);
    long long item = x.wide ? at[2] + n[0] : at[3] + n[1], slot = at[4] + n[2];
    Item* const items = x.wide ? items_w : items_n;
    int* const first = x.wide ? first_w : first_n;
    const long long most = x.wide ? s.max_items_w : s.max_items_n;
    long long r = p0 / run, edge = (r + 1) * run;  // the run that p0 lies in, its end
    for (int j = 0; j < x.n; ++j) {
      int nq, limit, len;
      x.at(p, j, nq, limit, len);
      const int k = pieces(p0, len);
      const bool direct = !sblocks && k == 1;
      const int groups = (nq + s.group - 1) / s.group;
      const long long b = blk + pos[2] + j;
      if (b < s.max_blocks) blocks[b] = BlockSlots{(int)slot, direct ? 0 : k, groups, 0};
      Item it{};
      it.flags = (x.shared ? kShared : 0) | (direct ? kDirect : 0);
      it.seq = x.shared ? 0 : e - lead;
      it.row0 = x.q.row0;
      it.q0 = (x.shared ? e : j) * x.block;  // an entry is one shared block
      it.nq = nq;
      it.limit = limit;
      it.len = x.shared ? limit : x.q.len;
      it.rows = x.q.rows;
      const long long t0 = p0 + ahead, p1 = t0 + len;  // position of the first tile, of the end
      for (long long q = p0; q < p1;) {
        const long long end = min(edge, p1);
        if (q == edge - run) first[r] = (int)item;  // r < the runs there are
        if (end > t0) {
          it.t0 = (int)max(q - t0, 0ll);
          it.t1 = (int)(end - t0);
          it.slot = (int)slot;
          if (!direct) slot += groups;
          if (item < most) items[item] = it;
          ++item;
        }
        q = end;
        if (q == edge) ++r, edge += run;
      }
      p0 = p1;
    }
    at[0] += tp[0];
    at[1] += tp[1];
    blk += tp[2];
    at[2] += tn[0];
    at[3] += tn[1];
    at[4] += tn[2];
  }
  __syncthreads();
  // runs behind the last item are empty
  for (int r = (int)((all[0] + len_w - 1) / len_w) + tid; r <= s.workers; r += kPlanThreads) first_w[r] = (int)at[2];
  for (int r = (int)((all[1] + len_n - 1) / len_n) + tid; r <= s.waves * s.workers; r += kPlanThreads)
    first_n[r] = (int)at[3];
  if (tid == 0) {
    const bool together = d.shared_workers + d.own_workers + d.narrow_workers > s.workers;
    head.rows = R;
    head.shared_block = sblocks ? sblock : 0;
    head.shared_items = (int)min((long long)shared_items, s.max_items_w);
    head.shared_workers = wblocks ? d.shared_workers : 0;
    head.own_first = together ? 0 : d.shared_workers;
    head.own_workers = d.own_workers;
    head.narrow_first = together ? 0 : d.shared_workers + d.own_workers;
    head.narrow_workers = s.waves ? d.narrow_workers : 0;
    *reinterpret_cast<PlanHead*>(plan) = head;
  }
}

// Where the parts of each query row lie.
__global__ __launch_bounds__(256) void plan_rows_kernel(Paged p, PlanShape s, uint8_t* plan) {
  const int x = blockIdx.x * 256 + threadIdx.x;
  const int R = rows_of(p);
  if (x >= R * p.G) return;
  const int r = x / p.G;
  int lo = 0, hi = p.n_seqs - 1;  // last b with row_start[b] <= r
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (p.row_start[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  const Seq q = seq_of(p, lo, R);
  const int rows = q.rows * p.G, at = x - q.row0 * p.G;
  RowSlots o{};
  if (at >= 0 && at < rows) {
    const int block = wide_rows(s, rows, keys_of(p, q)) ? s.wide : s.narrow;
    const long long blk = reinterpret_cast<const int*>(plan + s.off_seqs)[lo] + at / block;
    if (blk < s.max_blocks) {
      const BlockSlots d = reinterpret_cast<const BlockSlots*>(plan + s.off_blocks)[blk];
      const int in = at % block;
      o.part[1] = {d.slot + in / s.group, d.splits, d.groups, in % s.group};
    }
  }
  if (const int sb = reinterpret_cast<const PlanHead*>(plan)->shared_block) {
    const BlockSlots d = reinterpret_cast<const BlockSlots*>(plan + s.off_blocks)[x / sb];
    o.part[0] = {d.slot + x % sb / s.group, d.splits, d.groups, x % s.group};
  }
  reinterpret_cast<RowSlots*>(plan + s.off_rows)[x] = o;
}

// ------------------------------------------------------ attention, float32
__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// Keys and values in float32, and in 8 bits with a scale for the 16 rows of a
// tile: four elements as they are read, and as numbers.
struct Rows32 {
  using T = float;
  using Raw = f32x4;
  static __device__ __forceinline__ Raw read(const T* p) { return load4(p); }
  static __device__ __forceinline__ f32x4 get(Raw x, float) { return x; }
  using Args = PagedAttnArgs;
  static __device__ __forceinline__ float scale(const Args&, int, int, int, int) { return 1.f; }
};
struct Rows8 {
  using T = uint8_t;
  using Raw = uint32_t;
  static __device__ __forceinline__ Raw read(const T* p) { return *reinterpret_cast<const uint32_t*>(p); }
  static __device__ __forceinline__ f32x4 get(Raw x, float up) {
    float f[4];
    values4(x, up, f);
    return f32x4{f[0], f[1], f[2], f[3]};
  }
  using Args = PagedAttn8Args;
  static __device__ __forceinline__ float scale(const Args& a, int kv, int page, int g, int row) {
    return scale_of(a.c.scales[kv] + (long long)page * a.c.scale_stride + (long long)g * a.c.page_blocks +
                    row / kBlockRows);
  }
};

// One item of up to 16 query rows on the f32 matrix instruction (16x16x4).
// The keys go in tiles of 16, dealt round-robin to the waves; a wave computes
// S^T = K Q^T and O^T += V^T P^T with its own online softmax, and the waves
// merge through LDS.  No operand is staged: K and V are read in runs of 4
// columns straight into operand registers, and P is already in B-operand
// order (lane (c, q) holds row c's scores of keys 4q .. 4q + 3).  Lane (c, q)
// of the O^T accumulator dt holds row c, columns 64 (dt / 4) + 16 q + 4 r +
// dt % 4.  Bound by latency where it is used (float32 is the small option): 53
// rows of three tries over 128 + 100 tokens take 6.3 us.
template <int D, class C>
__global__ __launch_bounds__(64 * kF32Waves, f32_per_cu(D)) void paged_attn_f32_kernel(typename C::Args a) {
  constexpr int NW = kF32Waves;
  constexpr int KS = D / 16;
  __shared__ f32x4 o_s[NW][KS][64];
  __shared__ f32x2_t ml_s[NW][16];
  __shared__ int odd_s[NW];
  const Paged& p = a.p;
  const int g = blockIdx.x % p.Hkv, worker = blockIdx.x / p.Hkv;
  const PlanHead head = load_head(a);
  if (!plan_fits(head, a.want)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, qd = lane >> 4;
  each_wide(a, head, worker, [&](int item) {
    const Item it = load_item(a.plan + a.off_items_w, item);
    const bool on = c < it.nq;
    const int qi = it.q0 + min(c, it.nq - 1), i = qi / p.G, head_q = g * p.G + qi - i * p.G;
    const long long row = (long long)it.row0 + i;
    const Pages pages(p, it);
    const int head_off = g << p.page_shift, in_page = (1 << p.page_shift) - 1;
    using T = typename C::T;
    const T* const kp = (const T*)a.k;
    const T* const vp = (const T*)a.v;
    const int s0 = 4 * it.t0, s1 = min(4 * it.t1, (it.limit + 15) / 16);
    const int all = all_see(p, it);
    bool bad = false;

    f32x4 qv[KS];
    typename C::Raw kv[KS];
    float k_up = 1.f;
    const float* const qrow = (const float*)a.q + (row * p.Hq + head_q) * D + 4 * qd;
#pragma unroll
    for (int s = 0; s < KS; ++s) qv[s] = load4(qrow + 16 * s) * a.scale_log2e;
    // rows past the keys re-read the last one (weight zero)
    const auto tile_base = [&](int page, int t) {
      return (long long)page * p.page_stride + ((long long)head_off + ((16 * t) & in_page)) * D;
    };
    const auto load_k = [&](int t) {
      const int page = pages.at(16 * t, bad);
      const T* kr = kp + tile_base(page, t) + (size_t)min(c, it.limit - 1 - 16 * t) * D + 4 * qd;
#pragma unroll
      for (int s = 0; s < KS; ++s) kv[s] = C::read(kr + 16 * s);
      k_up = C::scale(a, 0, page, g, (16 * t) & in_page);
    };
    f32x4 o[KS];
#pragma unroll
    for (int dt = 0; dt < KS; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    if (s0 + wave < s1) load_k(s0 + wave);
    for (int t = s0 + wave; t < s1; t += NW) {
      const int lo = 16 * t;
      typename C::Raw vv[4][D / 64];
      const int page = pages.at(16 * t, bad);
      const T* const vb = vp + tile_base(page, t);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
          vv[r][h] = C::read(vb + (size_t)min(4 * qd + r, it.limit - 1 - lo) * D + 64 * h + 4 * c);
      const float v_up = C::scale(a, 1, page, g, (16 * t) & in_page);
      f32x4 score = {0.f, 0.f, 0.f, 0.f};
      // chains of eight products added in a tree: few roundings in a row
#pragma unroll
      for (int s = 0; s < KS; s += 4) {
        f32x4 sc[8], kk[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) kk[x] = C::get(kv[s + x], k_up);
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) sc[ch] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int ch = 0; ch < 8; ++ch) {
            const int x = s + ch / 2, e = 2 * (ch & 1) + j;
            sc[ch] = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[x - s][e], qv[x][e], sc[ch], 0, 0, 0);
          }
        score += ((sc[0] + sc[1]) + (sc[2] + sc[3])) + ((sc[4] + sc[5]) + (sc[6] + sc[7]));
      }
      if (t + NW < s1) load_k(t + NW);
      uint64_t mw = ~0ull;
      if (lo + 16 > all) mw = seen(p, it, i, (int)row, lo) >> (4 * qd);
      float pr[4], mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        pr[r] = (mw >> r) & 1ull ? score[r] : -INFINITY;
        mx = fmaxf(mx, pr[r]);
      }
      mx = fmaxf(mx, shfl_xor_f(mx, 16));
      mx = fmaxf(mx, shfl_xor_f(mx, 32));
      // the reference exponent is an integer: factors between tiles are powers
      // of two and round nothing
      const float m_new = fmaxf(m_run, ceilf(mx)), base = m_new == -INFINITY ? 0.f : m_new;
      if (__any(m_new > m_run)) {
        const float alpha = exp2f(m_run - base);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < KS; ++dt) o[dt] *= alpha;
        m_run = m_new;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) pr[r] = exp2f(pr[r] - base);
      l_run += (pr[0] + pr[1]) + (pr[2] + pr[3]);
      f32x4 vn[4][D / 64];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int h = 0; h < D / 64; ++h) vn[r][h] = C::get(vv[r][h], v_up);
#pragma unroll
      for (int dt = 0; dt < KS; ++dt) {
        f32x4 pv[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int r = 0; r < 4; ++r)
          pv[r & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(vn[r][dt >> 2][dt & 3], pr[r], pv[r & 1], 0, 0, 0);
        o[dt] += pv[0] + pv[1];
      }
    }
    l_run += shfl_xor_f(l_run, 16);
    l_run += shfl_xor_f(l_run, 32);
#pragma unroll
    for (int dt = 0; dt < KS; ++dt) o_s[wave][dt][lane] = o[dt];
    if (qd == 0) ml_s[wave][c] = f32x2_t{m_run, l_run};
    f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < KS; ++dt) zero += o[dt] * 0.f;
    const int odd = __any(!((zero[0] + zero[1]) + (zero[2] + zero[3]) == 0.f) && l_run < INFINITY);
    if (lane == 0) odd_s[wave] = (odd ? 1 : 0) | (__any(bad) ? 2 : 0);
    __syncthreads();
    float m = -INFINITY, den = 0.f;
    for (int w = 0; w < NW; ++w) m = fmaxf(m, ml_s[w][c][0]);
    const float base = m == -INFINITY ? 0.f : m;
    const bool poison = __any(lane < NW && (odd_s[lane < NW ? lane : 0] & 2));
    // A value of V that is not finite counts only for the query rows that give
    // its key a weight, but the matrix products multiply it by the zeros of the
    // others too, and zero times it is NaN.  So where a wave has a row of such
    // sums the block adds its keys once more, one by one and relative to the
    // rows' final exponents, without those of weight zero.  (Not for a row whose
    // weights are not finite: that is NaN either way.)
    if (__any(lane < NW && (odd_s[lane < NW ? lane : 0] & 1))) {
      __syncthreads();  // every wave has read ml_s and odd_s
      l_run = 0.f;
#pragma unroll
      for (int dt = 0; dt < KS; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int t = s0 + wave; t < s1; t += NW) {
        const int lo = 16 * t;
        const int page = pages.at(lo, bad);
        const long long tb = tile_base(page, t);
        const float ku = C::scale(a, 0, page, g, lo & in_page), vu = C::scale(a, 1, page, g, lo & in_page);
        const uint64_t mw = seen(p, it, i, (int)row, lo);
#pragma unroll 1
        for (int j = 0; j < 16 && lo + j < it.limit; ++j) {
          const T* kr = kp + tb + (size_t)j * D + 4 * qd;
          f32x4 s4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < KS; ++s) s4 += C::get(C::read(kr + 16 * s), ku) * (load4(qrow + 16 * s) * a.scale_log2e);
          float sc = (s4[0] + s4[1]) + (s4[2] + s4[3]);
          sc += shfl_xor_f(sc, 16);
          sc += shfl_xor_f(sc, 32);
          const float pk = (mw >> j) & 1ull ? exp2f(sc - base) : 0.f;
          if (pk == 0.f) continue;
          l_run += pk;
          const T* vr = vp + tb + (size_t)j * D + 16 * qd;
#pragma unroll
          for (int h = 0; h < D / 64; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const f32x4 x = C::get(C::read(vr + 64 * h + 4 * e), vu);
#pragma unroll
              for (int d4 = 0; d4 < 4; ++d4) o[4 * h + d4][e] += pk * x[d4];
            }
        }
      }
#pragma unroll
      for (int dt = 0; dt < KS; ++dt) o_s[wave][dt][lane] = o[dt];
      if (qd == 0) ml_s[wave][c] = f32x2_t{m, l_run};
      __syncthreads();
    }
    if (!on) return;
    float wgt[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const f32x2_t ml = ml_s[w][c];
      wgt[w] = exp2f(ml[0] - base);
      den += wgt[w] * ml[1];
    }
    if (poison) den = __builtin_nanf("");
    const float inv = den == 0.f ? 0.f : 1.f / den;  // a row that sees no key is zero
#pragma unroll
    for (int dt0 = 0; dt0 < KS; dt0 += NW) {  // a wave adds every fourth accumulator
      const int dt = dt0 + wave;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) acc += wgt[w] * o_s[w][dt][lane];
      if (it.flags & kDirect) {
        float* orow = (float*)a.out + (row * p.Hq + head_q) * D + 64 * (dt >> 2) + 16 * qd + (dt & 3);
#pragma unroll
        for (int r = 0; r < 4; ++r) orow[4 * r] = acc[r] * inv;
      } else if (it.slot < a.max_slots) {
        const size_t sl = (size_t)it.slot * p.Hkv + g;
        reinterpret_cast<f32x4*>(a.part_o)[(sl * KS + dt) * 64 + lane] = acc;
        if (dt == 0 && qd == 0) reinterpret_cast<f32x2_t*>(a.part_ml)[sl * 16 + c] = f32x2_t{m, den};
      }
    }
  });
}

// ------------------------------------------------------------------- join
// Adds the parts of every row.  A wave has one accumulator piece of a group of
// stacked query rows and KV head, and a lane 4 columns of one row over the
// row's shared and own slots.  Lane (c, q) of a piece holds row c and, in
// float32 (groups of 16), columns 64 (piece / 4) + 16 q + 4 e + piece % 4; in
// bf16 (groups of 32) columns 8 piece + 4 q + e.  Bound by latency: the plan's
// head and the row's slots are asked for together, then four slots at a time:
// 5 us for 64 rows of 32 heads, 7 for 385.  Few rows may be split over hundreds
// of slots; then four waves share a piece's (PAR), eight slots at a time each:
// the call for one row of 32 heads over a 22k prompt takes 42 us, 120 with one,
// for two rows 33 and 94.  More rows have few parts, and four times the waves
// cost more: 56 us, not 44, for 1145 rows of four prompts.  Hence the bound on
// the workgroups in launch_attn.
template <class T, int D, int PAR>
__global__ __launch_bounds__(256) void join_kernel(PagedAttnArgs a) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int GR = BF ? 32 : 16, NP = D * GR / 256;
  constexpr int AT_ONCE = PAR == 1 ? 4 : 8, PIECES = 4 / PAR;  // of a workgroup
  const Paged& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane % GR, qd = lane / GR;
  const int w = blockIdx.x / (NP / PIECES), pc = PIECES * (blockIdx.x % (NP / PIECES)) + wave % PIECES;
  const int share = wave / PIECES;
  const int g = w % p.Hkv, x = (w / p.Hkv) * GR + c;
  const int i = x / p.G, h = g * p.G + x - i * p.G;
  const PlanHead head = load_head(a);
  const RowSlots rs = reinterpret_cast<const RowSlots*>(a.plan + a.off_rows)[min(x, p.n_rows * p.G - 1)];
  const bool fits = plan_fits(head, a.want);
  const bool in = i < (fits ? head.rows : min(p.row_start[p.n_seqs], p.n_rows));
  T* const orow = (T*)a.out + ((size_t)i * p.Hq + h) * D;
  const auto put = [&](f32x4 o) {
    if constexpr (BF)
      *reinterpret_cast<u32x2*>(orow + 8 * pc + 4 * qd) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) orow[64 * (pc >> 2) + 16 * qd + 4 * e + (pc & 3)] = o[e];
  };
  if (!fits) {
    const float nan = __builtin_nanf("");
    if (in && share == 0) put(f32x4{nan, nan, nan, nan});
    return;
  }
  const int n0 = rs.part[0].splits;
  const int n = in && rs.part[1].splits > 0 ? n0 + rs.part[1].splits : 0;  // 0: written by its item
  float m = -INFINITY, den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  // adds N parts with their maxima and sums
  const auto add = [&](auto& ms, auto& dens, auto& os) {
    constexpr int N = sizeof(ms) / sizeof(float);
    float mn = m;
#pragma unroll
    for (int k = 0; k < N; ++k) mn = fmaxf(mn, ms[k]);
    const float base = mn == -INFINITY ? 0.f : mn;
    const float wa = exp2f(m - base);
    den *= wa;
    acc *= wa;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float wb = exp2f(ms[k] - base);
      den += dens[k] * wb;
      if (wb > 0.f) acc += os[k] * wb;  // zero times an infinite sum is not zero
    }
    m = mn;
  };
  for (int s = share * AT_ONCE; s < n; s += PAR * AT_ONCE) {
    float ms[AT_ONCE], dens[AT_ONCE];
    f32x4 o[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {  // past the last one: that again, without weight
      const int t = min(s + k, n - 1);
      const RowSlots::Part& r = rs.part[t < n0 ? 0 : 1];
      const long long slot = r.slot + (long long)(t < n0 ? t : t - n0) * r.stride;
      const size_t sl = (size_t)min(slot, a.max_slots - 1) * p.Hkv + g;
      const f32x2_t ml = reinterpret_cast<const f32x2_t*>(a.part_ml)[sl * GR + r.row];
      o[k] = reinterpret_cast<const f32x4*>(a.part_o)[(sl * NP + pc) * 64 + GR * qd + r.row];
      ms[k] = s + k < n ? ml[0] : -INFINITY;
      dens[k] = s + k < n ? ml[1] : 0.f;
    }
    add(ms, dens, o);
  }
  if constexpr (PAR > 1) {
    __shared__ float ms_s[PAR][64], den_s[PAR][64];
    __shared__ f32x4 o_s[PAR][64];
    ms_s[share][lane] = m, den_s[share][lane] = den, o_s[share][lane] = acc;
    __syncthreads();
    if (share > 0) return;
    float ms[PAR - 1], dens[PAR - 1];
    f32x4 o[PAR - 1];
#pragma unroll
    for (int k = 0; k < PAR - 1; ++k) ms[k] = ms_s[k + 1][lane], dens[k] = den_s[k + 1][lane], o[k] = o_s[k + 1][lane];
    add(ms, dens, o);
  }
  if (n > 0) put(acc * (den == 0.f ? 0.f : 1.f / den));
}

template <class T, int D>
void launch_attn(const PagedAttn8Args& a, const PlanShape& s, bool eight, bool neg, hipStream_t st) {
  const unsigned items = (unsigned)(s.workers * a.p.Hkv);
  if constexpr (sizeof(T) == 2) {
    if (eight && neg) paged_attn8_kernel<D, true><<<items, 64 * kPagedWaves, 0, st>>>(a);
    else if (eight) paged_attn8_kernel<D, false><<<items, 64 * kPagedWaves, 0, st>>>(a);
    else if (neg) paged_attn_bf16_kernel<D, true><<<items, 64 * kPagedWaves, 0, st>>>(a);
    else paged_attn_bf16_kernel<D, false><<<items, 64 * kPagedWaves, 0, st>>>(a);
  } else {
    if (eight) paged_attn_f32_kernel<D, Rows8><<<items, 64 * kF32Waves, 0, st>>>(a);
    else paged_attn_f32_kernel<D, Rows32><<<items, 64 * kF32Waves, 0, st>>>(a);
  }
  const long long groups = ((long long)a.p.n_rows * a.p.G + s.group - 1) / s.group;
  const long long blocks = groups * a.p.Hkv * (D * s.group / 1024);
  if (blocks <= 2 * device_cus()) join_kernel<T, D, 4><<<(unsigned)(4 * blocks), 256, 0, st>>>(a);
  else join_kernel<T, D, 1><<<(unsigned)blocks, 256, 0, st>>>(a);
}

size_t workspace_bytes(const ooo_paged_batch& b, const PlanShape& s) {
  return (size_t)s.max_slots * b.n_kv_heads * s.group * (b.head_dim + 2) * sizeof(float);
}

int make_plan(const char* who, const ooo_paged_batch* batch, const Paged& p, bool eight, void* plan,
              size_t plan_bytes, void* stream) {
  OOO_REQUIRE(plan, OOO_ERR_INVALID, "%s: null pointer", who);
  OOO_REQUIRE(aligned16(plan), OOO_ERR_UNSUPPORTED, "%s: plan is not 16-byte aligned", who);
  const PlanShape s = plan_shape(*batch);
  OOO_REQUIRE(plan_grid_ok(*batch, s), OOO_ERR_UNSUPPORTED, "%s: more than 2^30 workgroups", who);
  OOO_REQUIRE(plan_bytes >= (size_t)s.bytes, OOO_ERR_CAPACITY, "%s: plan of %lld bytes needed (got %zu)", who,
              s.bytes, plan_bytes);
  PlanHead head{};
  plan_key(*batch, eight, head.key);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  plan_kernel<<<1, kPlanThreads, 0, st>>>(p, s, eight ? kCosts8 : kCosts, head, batch->head_dim == 64,
                                          (uint8_t*)plan);
  const long long q = (long long)p.n_rows * p.G;
  plan_rows_kernel<<<(unsigned)((q + 255) / 256), 256, 0, st>>>(p, s, (uint8_t*)plan);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ooo::ok();
}

// a: with the batch, and the cache where it is one of 8 bits.
int attend(const char* who, const ooo_paged_batch* batch, PagedAttn8Args& a, bool eight, const void* plan,
           size_t plan_bytes, const void* q, const void* k_pages, const void* v_pages, float scale, void* out,
           void* workspace, size_t ws_bytes, void* stream) {
  OOO_REQUIRE(plan && q && k_pages && v_pages && out && workspace, OOO_ERR_INVALID, "%s: null pointer", who);
  OOO_REQUIRE(aligned16(plan) && aligned16(q) && aligned16(k_pages) && aligned16(v_pages) && aligned16(out) &&
                  aligned16(workspace),
              OOO_ERR_UNSUPPORTED, "%s: a pointer is not 16-byte aligned", who);
  const float scale_log2e = scale * 1.4426950408889634f;
  OOO_REQUIRE(fabsf(scale_log2e) < INFINITY, OOO_ERR_INVALID, "%s: scale %g is not finite in base 2", who,
              (double)scale);
  const PlanShape s = plan_shape(*batch);
  OOO_REQUIRE(plan_grid_ok(*batch, s), OOO_ERR_UNSUPPORTED, "%s: more than 2^30 workgroups", who);
  OOO_REQUIRE(plan_bytes >= (size_t)s.bytes, OOO_ERR_CAPACITY, "%s: plan of %lld bytes needed (got %zu)", who,
              s.bytes, plan_bytes);
  const size_t need = workspace_bytes(*batch, s);
  OOO_REQUIRE(ws_bytes >= need, OOO_ERR_CAPACITY, "%s: workspace of %zu bytes needed (got %zu)", who, need,
              ws_bytes);
  plan_key(*batch, eight, a.want.key);
  a.plan = (const uint8_t*)plan;
  a.off_first_w = s.off_first_w;
  a.off_first_n = s.off_first_n;
  a.off_items_w = s.off_items_w;
  a.off_items_n = s.off_items_n;
  a.off_rows = s.off_rows;
  a.max_items_w = (int)s.max_items_w;
  a.max_items_n = (int)s.max_items_n;
  a.workers = s.workers;
  a.q = q;
  a.k = k_pages;
  a.v = v_pages;
  a.out = out;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + (size_t)s.max_slots * batch->n_kv_heads * s.group * batch->head_dim;
  a.max_slots = s.max_slots;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool bf = batch->dt == OOO_BF16, wide = batch->head_dim == 128;
  a.scale_log2e = scale_log2e;
  if (bf) {
    // The bf16 kernel scales scores that are -inf where a key is not seen: by a
    // positive number.  In place of 0 the least one, 2^-149, which moves weights
    // by less than 2^-21 of themselves.
    a.scale_log2e = fmaxf(fabsf(scale_log2e), 0x1p-149f);
  }
  const bool neg = scale_log2e < 0.f;
  if (bf && wide) launch_attn<uint16_t, 128>(a, s, eight, neg, st);
  else if (bf) launch_attn<uint16_t, 64>(a, s, eight, neg, st);
  else if (wide) launch_attn<float, 128>(a, s, eight, neg, st);
  else launch_attn<float, 64>(a, s, eight, neg, st);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ooo::ok();
}

}  // namespace
}  // namespace ooo

using namespace ooo;

extern "C" size_t ooo_paged_plan_bytes(const ooo_paged_batch* batch) {
  Paged p{};
  if (check_paged("ooo_paged_plan_bytes", batch, p) != OOO_OK) return 0;
  return (size_t)plan_shape(*batch).bytes;
}

extern "C" int ooo_paged_plan(const ooo_paged_batch* batch, void* plan, size_t plan_bytes, void* stream) {
  Paged p{};
  const int rc = check_paged("ooo_paged_plan", batch, p);
  if (rc != OOO_OK) return rc;
  return make_plan("ooo_paged_plan", batch, p, false, plan, plan_bytes, stream);
}

extern "C" size_t ooo_paged_attn_workspace(const ooo_paged_batch* batch) {
  Paged p{};
  if (check_paged("ooo_paged_attn_workspace", batch, p) != OOO_OK) return 0;
  return workspace_bytes(*batch, plan_shape(*batch));
}

extern "C" int ooo_paged_attn(const ooo_paged_batch* batch, const void* plan, size_t plan_bytes, const void* q,
                              const void* k_pages, const void* v_pages, float scale, void* out, void* workspace,
                              size_t ws_bytes, void* stream) {
  PagedAttn8Args a{};
  const int rc = check_paged("ooo_paged_attn", batch, a.p);
  if (rc != OOO_OK) return rc;
  return attend("ooo_paged_attn", batch, a, false, plan, plan_bytes, q, k_pages, v_pages, scale, out, workspace,
                ws_bytes, stream);
}

extern "C" size_t ooo_paged_plan8_bytes(const ooo_paged_batch* batch) {
  Paged p{};
  Cache8 c{};
  if (check_cache8("ooo_paged_plan8_bytes", batch, nullptr, p, c) != OOO_OK) return 0;
  return (size_t)plan_shape(*batch).bytes;
}

extern "C" int ooo_paged_plan8(const ooo_paged_batch* batch, void* plan, size_t plan_bytes, void* stream) {
  Paged p{};
  Cache8 c{};
  const int rc = check_cache8("ooo_paged_plan8", batch, nullptr, p, c);
  if (rc != OOO_OK) return rc;
  return make_plan("ooo_paged_plan8", batch, p, true, plan, plan_bytes, stream);
}

extern "C" size_t ooo_paged_attn8_workspace(const ooo_paged_batch* batch) {
  Paged p{};
  Cache8 c{};
  if (check_cache8("ooo_paged_attn8_workspace", batch, nullptr, p, c) != OOO_OK) return 0;
  return workspace_bytes(*batch, plan_shape(*batch));
}

extern "C" int ooo_paged_attn8(const ooo_paged_batch* batch, const ooo_cache8* cache, int32_t layer,
                               const void* plan, size_t plan_bytes, const void* q, float scale, void* out,
                               void* workspace, size_t ws_bytes, void* stream) {
  const char* const who = "ooo_paged_attn8";
  PagedAttn8Args a{};
  OOO_REQUIRE(cache, OOO_ERR_INVALID, "%s: cache is null", who);
  int rc = check_cache8(who, batch, cache, a.p, a.c);
  if (rc == OOO_OK) rc = take_layer(who, cache, layer, a.c);
  if (rc != OOO_OK) return rc;
  return attend(who, batch, a, true, plan, plan_bytes, q, a.c.pages[0], a.c.pages[1], scale, out, workspace, ws_bytes,
                stream);
}
