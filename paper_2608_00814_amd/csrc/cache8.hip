// Rows of a batch into, inside and between cache pages of 8-bit numbers, and
// sequences that continue another one's cache of any type.
//
//  * ooo_paged_append8   per-head RMSNorm of q and k, rotation at the row's
//                        position, q to [rows][Hq][D], k and v quantised into
//                        the pages, block by block
//  * ooo_paged_compact8  the accepted rows of every sequence moved together
//  * ooo_paged_fork(8)   page tables by reference, the open page by copy
#include "cache8.h"
#include "rope.h"
#include "vec16.h"

#include <algorithm>

namespace ooo {
namespace {

// ----------------------------------------------------------------- append
constexpr int kAppendWaves = 4;
constexpr int kFewRows = 4096;  // up to so many, a block's heads are shared out
// Rows of a workgroup of the pages' part where sequences bring several (a block
// of 32 begins in at most two of them); one row each where most bring one.
constexpr int kSpan = 8;

// The place of a new row (0 <= r < R: rows_of): its sequence, index in it, own
// token and page (-1: it has none).
struct Place {
  int i, rows, len, page, pos;
  long long slot;
};
__device__ __forceinline__ Place place_of(const Paged& p, int r, int R, const int32_t* depth, int lane) {
  Place o;
  const int b = __builtin_amdgcn_readfirstlane(seq_of_row(p.row_start, p.n_seqs, r, lane));
  const Seq q = seq_of(p, b, R);
  o.len = p.seq_len[b];
  o.i = r - q.row0;
  o.rows = q.rows;
  o.slot = (long long)o.len + o.i;
  o.pos = p.shared_len + o.len + (depth ? depth[r] : o.i);
  const bool ok = o.len >= 0 && o.i >= 0 && o.i < o.rows && o.slot < p.own_cap;
  o.page = ok ? p.table[(size_t)b * p.table_ld + (o.slot >> p.page_shift)] : -1;
  if (o.page >= p.n_pages) o.page = -1;
  return o;
}

// A lane's share of a head's row: N elements of each half.
template <class T>
struct Half {
  static constexpr int N = Vec16<T>::N;
  u32x4 a, c;
  __device__ __forceinline__ void load(const T* src, int half) {
    a = ld16(src);
    c = ld16(src + half);
  }
};

// Norm (over the head's LPH neighbouring lanes) and rotation of one head's row:
// x <- x / sqrt(mean(x^2) + eps) w, then the rotate-half pairs (x_j, x_{j+D/2}).
template <class T, int D>
__device__ __forceinline__ void norm_turn(float (&a)[Vec16<T>::N], float (&c)[Vec16<T>::N], const T* nw, float eps,
                                          int j0, const float* cs, const float* sn) {
  using V = Vec16<T>;
  constexpr int N = V::N, HALF = D / 2, LPH = HALF / N;
  if (nw) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) ss = __builtin_fmaf(a[e], a[e], __builtin_fmaf(c[e], c[e], ss));
#pragma unroll
    for (int off = LPH / 2; off > 0; off >>= 1) ss += shfl_xor_f(ss, off);
    const float rs = 1.f / sqrtf(ss / (float)D + eps);
    float wa[N], wc[N];
    V::unpack(ld16(nw + j0), wa);
    V::unpack(ld16(nw + HALF + j0), wc);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      a[e] = a[e] * rs * wa[e];
      c[e] = c[e] * rs * wc[e];
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float ra = a[e] * cs[j0 + e] - c[e] * sn[j0 + e], rc = c[e] * cs[j0 + e] + a[e] * sn[j0 + e];
    a[e] = ra;
    c[e] = rc;
  }
}

template <int N>
__device__ __forceinline__ void put_codes(uint8_t* dst, const float (&x)[N], float down) {
  if constexpr (N == 8) {
    *reinterpret_cast<u32x2*>(dst) =
        u32x2{codes4(x[0], x[1], x[2], x[3], down), codes4(x[4], x[5], x[6], x[7], down)};
  } else {
    *reinterpret_cast<uint32_t*>(dst) = codes4(x[0], x[1], x[2], x[3], down);
  }
}

struct AppendArgs {
  Paged p;
  Cache8 c;
  const void *qkv, *q_norm, *k_norm;
  long long ld;
  float eps;
  const int32_t* depth;
  void* q_out;
  int span;  // rows of a workgroup of the pages' part
  RopeFreq fr;
};

// One workgroup's share of the queries: a row a wave for the angles (lane j
// computes pair j's, in double), then head groups a wave for all four rows.
template <class T, int D>
__device__ __forceinline__ void append_queries(const AppendArgs& a, int r0, int lane, int wave, float* cs_s,
                                               float* sn_s) {
  using V = Vec16<T>;
  constexpr int N = V::N, HALF = D / 2, LPH = HALF / N, HPW = 64 / LPH;
  __shared__ int on_s[kAppendWaves];
  const Paged& p = a.p;
  const int R = rows_of(p);
  const int r = r0 + wave;
  bool in = r < R;
  if (in) {
    const Place at = place_of(p, r, R, a.depth, lane);
    in = at.i >= 0 && at.i < at.rows;
    if (lane < HALF) rope_sincos(at.pos, a.fr.f[lane], sn_s[wave * HALF + lane], cs_s[wave * HALF + lane]);
  }
  if (lane == 0) on_s[wave] = in;
  __syncthreads();
  const int j0 = (lane % LPH) * N;
  for (int h0 = wave * HPW; h0 < p.Hq; h0 += kAppendWaves * HPW) {
    const int h = h0 + lane / LPH;
    Half<T> x[kAppendWaves];
#pragma unroll
    for (int k = 0; k < kAppendWaves; ++k)
      if (on_s[k]) x[k].load((const T*)a.qkv + (size_t)(r0 + k) * a.ld + (size_t)min(h, p.Hq - 1) * D + j0, HALF);
#pragma unroll
    for (int k = 0; k < kAppendWaves; ++k) {
      if (!on_s[k]) continue;
      float lo[N], hi[N];
      V::unpack(x[k].a, lo);
      V::unpack(x[k].c, hi);
      norm_turn<T, D>(lo, hi, (const T*)a.q_norm, a.eps, j0, cs_s + k * HALF, sn_s + k * HALF);
      if (h < p.Hq) {
        T* const dst = (T*)a.q_out + ((size_t)(r0 + k) * p.Hq + h) * D + j0;
        st16(dst, V::pack(lo));
        st16(dst + HALF, V::pack(hi));
      }
    }
  }
}

// The new rows r0 .. r0 + m - 1 of one sequence that lie in one block, at block
// row `row` of block `blk` of the page.  A wave takes one head's K or V (task
// kv Hkv + g): its rows (8 or 4 at a time) stay in registers while their largest
// size, and so the scale, is found.  One row alone (decoding): a wave takes as
// many heads at once (task kv groups + group).  `held`: block rows below `row`
// that are committed.
template <class T, int D>
__device__ __forceinline__ void append_block(const AppendArgs& a, int task, int r0, int m, int page, int blk, int row,
                                             bool held, int lane, const float* cs_s, const float* sn_s) {
  using V = Vec16<T>;
  constexpr int N = V::N, HALF = D / 2, LPH = HALF / N, SLOTS = 64 / LPH, STEPS = kBlockRows / SLOTS;
  const Paged& p = a.p;
  const int j0 = (lane % LPH) * N, s = lane / LPH;
  const auto load = [&](Half<T>& x, int i, int g, int kv) {
    x.load((const T*)a.qkv + (size_t)(r0 + i) * a.ld + (size_t)(p.Hq + kv * p.Hkv + g) * D + j0, HALF);
  };
  const auto row_at = [&](int kv, int g, int i) {  // block row i of head g
    return a.c.pages[kv] + (long long)page * p.page_stride +
           (((long long)g << p.page_shift) + blk * kBlockRows + i) * D;
  };
  const auto scale_at = [&](int kv, int g) {
    return a.c.scales[kv] + (long long)page * a.c.scale_stride + (long long)g * a.c.page_blocks + blk;
  };
  // puts the committed rows of a block of head g under a scale 2^k times theirs
  const auto regrade = [&](int kv, int g, int k) {
    for (int e = lane * 16; e < row * D; e += 64 * 16) {
      u32x4* const at = reinterpret_cast<u32x4*>(row_at(kv, g, 0) + e);
      u32x4 w = *at;
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = fewer4(w[x], k);
      *at = w;
    }
  };
  if (m == 1) {
    const int groups = (p.Hkv + SLOTS - 1) / SLOTS;
    const int kv = task >= groups, g0 = (task - kv * groups) * SLOTS, g = g0 + s;
    Half<T> x;
    load(x, 0, min(g, p.Hkv - 1), kv);
    const int was = held ? (int)*scale_at(kv, min(g, p.Hkv - 1)) - 127 : kLeastExp;
    float lo[N], hi[N];
    V::unpack(x.a, lo);
    V::unpack(x.c, hi);
    if (kv == 0) norm_turn<T, D>(lo, hi, (const T*)a.k_norm, a.eps, j0, cs_s, sn_s);
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, fmaxf(size_of(lo[e]), size_of(hi[e])));
#pragma unroll
    for (int off = LPH / 2; off > 0; off >>= 1) most = fmaxf(most, shfl_xor_f(most, off));
    const int exp = max(exp_for(most), was);
    if (g < p.Hkv) {
      uint8_t* const dst = row_at(kv, g, row) + j0;
      put_codes<N>(dst, lo, pow2(-exp));
      put_codes<N>(dst + HALF, hi, pow2(-exp));
      if (lane % LPH == 0 && (!held || exp != was)) *scale_at(kv, g) = (uint8_t)(exp + 127);
    }
    if (held)
      for (int y = 0; y < min(SLOTS, p.Hkv - g0); ++y) {
        const int k = __builtin_amdgcn_readlane(exp - was, y * LPH);
        if (k > 0) regrade(kv, g0 + y, k);
      }
    return;
  }
  const int kv = task >= p.Hkv, g = task - kv * p.Hkv;
  Half<T> x[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) load(x[k], min(k * SLOTS + s, m - 1), g, kv);
  const int was = held ? (int)*scale_at(kv, g) - 127 : kLeastExp;
  float lo[STEPS][N], hi[STEPS][N], most = 0.f;
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    V::unpack(x[k].a, lo[k]);
    V::unpack(x[k].c, hi[k]);
    const int i = min(k * SLOTS + s, m - 1);
    if (kv == 0) norm_turn<T, D>(lo[k], hi[k], (const T*)a.k_norm, a.eps, j0, cs_s + i * HALF, sn_s + i * HALF);
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, fmaxf(size_of(lo[k][e]), size_of(hi[k][e])));
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, shfl_xor_f(most, off));
  const int exp = max(exp_for(most), was);
  const float down = pow2(-exp);
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i = k * SLOTS + s;
    if (i >= m) continue;
    uint8_t* const dst = row_at(kv, g, row + i) + j0;
    put_codes<N>(dst, lo[k], down);
    put_codes<N>(dst + HALF, hi[k], down);
  }
  if (lane == 0 && (!held || exp != was)) *scale_at(kv, g) = (uint8_t)(exp + 127);
  if (held && exp > was) regrade(kv, g, exp - was);
}

// Workgroups blockIdx.x < `units` go over the rows from span blockIdx.x on and
// quantise the blocks that begin there (with a sequence's first new row, or a
// block of its own tokens); the others take four rows of queries each.  Up to
// kFewRows rows a block's heads go to several workgroups (blockIdx.y), four
// heads' K or V each: with 32 heads of 128 and 8 of K and V, 614 rows of four
// prompts take 12 us so and 20 with all heads in one, 2463 rows 21 and 25, 3197 of
// eight 23 and 25, 4914 42 and 40, 6399 47 and 42, 11760 of sixteen 70 and 65; with
// 2 heads of K and V no less or more.  (A row each of 1024 requests takes 18 so and
// 13 with all in one, of 3000 45 and 28: workgroups that find nothing to do.  Of 64,
// 6 either way.)  11760 rows of prompts: 63 us (264 MB, 4.2 TB/s of the 4.96 of a
// copy), the queries' part alone 43 and the pages' alone 33.  A row for each of 256
// requests: 5.9 us in a graph, 17.7 where every block's scale grows.
template <class T, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void append8_kernel(AppendArgs a, int units) {
  constexpr int HALF = D / 2, SLOTS = 64 / (HALF / Vec16<T>::N);
  __shared__ __attribute__((aligned(16))) float cs_s[kBlockRows * HALF], sn_s[kBlockRows * HALF];
  const Paged& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= units) {
    if (blockIdx.y == 0)
      append_queries<T, D>(a, ((int)blockIdx.x - units) * kAppendWaves, lane, wave, cs_s, sn_s);
    return;
  }
  const int R = rows_of(p);
  const int end = min(((int)blockIdx.x + 1) * a.span, R), first = (int)blockIdx.y * kAppendWaves;
  const int stride = (int)gridDim.y * kAppendWaves;
  for (int r = (int)blockIdx.x * a.span; r < end;) {
    const Place at = place_of(p, r, R, nullptr, lane);
    if (at.i < 0 || at.i >= at.rows || at.len < 0 || at.slot >= p.own_cap) {
      ++r;  // no sequence's row, or no place
      continue;
    }
    const int row = (int)(at.slot & (kBlockRows - 1));
    const int m = min(kBlockRows - row, at.rows - at.i);
    const int keys = m == 1 ? (p.Hkv + SLOTS - 1) / SLOTS : p.Hkv;  // tasks of K; as many of V
    if ((at.i == 0 || row == 0) && at.page >= 0 && first < 2 * keys) {
      const int blk = (int)(at.slot & ((1 << p.page_shift) - 1)) / kBlockRows;
      if (first < keys) {
        __syncthreads();  // the last block's angles are read
        for (int e = threadIdx.x; e < m * HALF; e += 64 * kAppendWaves) {
          const int i = e / HALF;
          const int pos = p.shared_len + at.len + (a.depth ? a.depth[r + i] : at.i + i);
          rope_sincos(pos, a.fr.f[e % HALF], sn_s[e], cs_s[e]);
        }
        __syncthreads();
      }
      for (int t = first + wave; t < 2 * keys; t += stride)
        append_block<T, D>(a, t, r, m, at.page, blk, row, at.i == 0 && row > 0, lane, cs_s, sn_s);
    }
    r += m;
  }
}

struct AppendGrid {
  long long units, rows;  // workgroups of the pages' part and of the queries'
};
AppendGrid append_grid(const AppendArgs& a) {
  const long long n = a.p.n_rows;
  return {(n + a.span - 1) / a.span, (n + kAppendWaves - 1) / kAppendWaves};
}

template <class T, int D>
void launch_append8(AppendArgs& a, hipStream_t st) {
  const int units = (int)append_grid(a).units, rows = (int)append_grid(a).rows;
  const int tasks = a.p.n_rows > kFewRows ? 1 : (2 * a.p.Hkv + kAppendWaves - 1) / kAppendWaves;
  append8_kernel<T, D><<<dim3(units + rows, tasks), 64 * kAppendWaves, 0, st>>>(a, units);
}

// ----------------------------------------------------------------- compact
// A workgroup has one layer and sequence and, a wave each, four of its heads' K
// or V.  A chain of dependent reads is the most of its time: path and page of 256
// rows are looked up once, a row a thread.  Then a wave takes the blocks that rows
// come into, the lowest first, a lane 16 numbers of a row, and reads all rows of
// a block before it writes one: since path[d] >= d rises strictly, later blocks'
// rows come from none that it wrote.  Rows that stay where they are (committed
// ones, the root) are read only if their scale grows.  (Two blocks at a time take
// 90 registers: 64 sequences of 8 rows in 36 layers took 29 us so, 21 like this.)
constexpr int kMapRows = 256;

template <int D>
__global__ __launch_bounds__(256) void compact8_kernel(Paged p, Cache8 c, long long layer_stride,
                                                       long long scale_layer_stride,
                                                       const int32_t* __restrict__ path,
                                                       const int32_t* __restrict__ accept, int path_cap) {
  constexpr int TPR = D / 16, RPS = 64 / TPR, STEPS = kBlockRows / RPS;
  __shared__ int page_s[kMapRows], row_s[kMapRows];  // where a row's numbers come from (-1: no row comes)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int task = (int)blockIdx.x * 4 + wave, b = blockIdx.y, g = task >> 1, kv = task & 1;
  const int len = p.seq_len[b], accepted = accept[b], rows = seq_of(p, b, rows_of(p)).rows;
  if (accepted < 0 || accepted >= path_cap || len < 0 || len >= p.own_cap) return;
  const int L = min(accepted, rows - 1);
  const int row0 = lane / TPR, sub = lane % TPR, in_page = (1 << p.page_shift) - 1;
  const auto page_of = [&](int token) {
    if (token < 0 || token >= p.own_cap) return -1;
    const int page = p.table[(size_t)b * p.table_ld + (token >> p.page_shift)];
    return page < p.n_pages ? page : -1;
  };
  const auto row_at = [&](int page, int row) {
    return c.pages[kv] + (long long)blockIdx.z * layer_stride + (long long)page * p.page_stride +
           (((long long)g << p.page_shift) + row) * D + sub * 16;
  };
  const auto scale_at = [&](int page, int row) {
    return c.scales[kv] + (long long)blockIdx.z * scale_layer_stride + (long long)page * c.scale_stride +
           (long long)g * c.page_blocks + row / kBlockRows;
  };
  for (int map0 = len / kBlockRows * kBlockRows; L >= 0 && map0 <= len + L; map0 += kMapRows) {
    {
      const int token = map0 + (int)threadIdx.x, d = token - len;
      int from = d < 0 ? token : -1;
      if (d >= 0 && d <= L) {
        const int i = path[(size_t)b * path_cap + d];
        if (i >= 0 && i < rows) from = len + i;
      }
      const int to = page_of(token);
      page_s[threadIdx.x] = from == token ? to : to >= 0 ? page_of(from) : -1;
      row_s[threadIdx.x] = from & in_page;
    }
    __syncthreads();
    for (int at = 0; g < p.Hkv && at < kMapRows && map0 + at <= len + L; at += kBlockRows) {
      const int first = map0 + at, to = page_of(first);  // the same in the whole wave
      int page[STEPS], row[STEPS], e[STEPS], most = -1000;
      bool stays[STEPS], moved = false;
      u32x4 w[STEPS];
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int x = s * RPS + row0;
        page[s] = page_s[at + x];
        row[s] = row_s[at + x];
        stays[s] = page[s] == to && row[s] == ((first + x) & in_page);
        e[s] = -1000;
        if (page[s] >= 0) {
          e[s] = (int)*scale_at(page[s], row[s]) - 127;
          if (!stays[s]) w[s] = ld16(row_at(page[s], row[s]));
          moved = moved || first + x >= len;
        }
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // all rows are here
#pragma unroll
      for (int s = 0; s < STEPS; ++s) most = max(most, e[s]);
#pragma unroll
      for (int off = 32; off >= TPR; off >>= 1) most = max(most, shfl_xor_i(most, off));
      if (!__any(moved)) continue;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int into = (first + s * RPS + row0) & in_page;
        if (page[s] < 0 || (stays[s] && e[s] == most)) continue;
        if (stays[s]) w[s] = ld16(row_at(to, into));
        if (e[s] != most)
#pragma unroll
          for (int x = 0; x < 4; ++x) w[s][x] = fewer4(w[s][x], most - e[s]);
        st16(row_at(to, into), w[s]);
      }
      if (lane == 0) *scale_at(to, first & in_page) = (uint8_t)(most + 127);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------- fork
struct ForkArgs {
  const int32_t* seq_len;
  const int32_t* table;
  const int32_t* parent;
  const int32_t* fresh;
  int32_t* len_out;
  int32_t* table_out;
  uint8_t* pages[2];
  uint8_t* scales[2];
  long long page_bytes, layer_bytes, scale_stride, scale_layer;
  int n_seqs, table_ld, page_shift, n_pages, own_cap, row_bytes, page_blocks;  // page_blocks 0: no scales
  int heads, heads_each;
};

// One workgroup for each layer, sequence, K or V and as many heads as have 32 KiB
// of a page (a workgroup a head took 42 us for 64 pages of 16 rows in 36 layers, by
// the number of workgroups alone, and takes 16 so); the first of a sequence writes
// its length and table.  Copies go past the caches; parents' rows, which their
// other children read too, do not: 64 children of 8 requests, pages of 64 rows of 8
// bits, 36 layers, take 28 us (130 MB written, 4.7 TB/s) and took 42 with ordinary
// stores, 45 with reads past the caches as well.
__global__ __launch_bounds__(256) void fork_kernel(ForkArgs a) {
  const int b = blockIdx.y, g0 = (int)(blockIdx.x >> 1) * a.heads_each, kv = blockIdx.x & 1;
  const int heads = min(a.heads_each, a.heads - g0);
  const bool in_place = a.len_out == a.seq_len, first = blockIdx.x == 0 && blockIdx.z == 0;
  const int p = a.parent[b];
  bool forks = p >= 0 && p != b && p < a.n_seqs;
  int n = 0, page = 0, to = 0, rows = 0;
  if (forks) {
    to = a.fresh[b];
    n = a.seq_len[p];
    const int pp = a.parent[p];
    rows = n & ((1 << a.page_shift) - 1);
    forks = to >= 0 && to < a.n_pages && n >= 0 && n < a.own_cap &&
            !(in_place && pp >= 0 && pp != p && pp < a.n_seqs);
    if (forks && rows > 0) {
      page = a.table[(size_t)p * a.table_ld + (n >> a.page_shift)];
      forks = page >= 0 && page < a.n_pages;
    }
  }
  if (first && (forks || !in_place)) {
    const int full = forks ? n >> a.page_shift : 0;
    for (int t = threadIdx.x; t < a.table_ld; t += 256) {
      const int x = forks && t == full ? to : a.table[(size_t)(t < full ? p : b) * a.table_ld + t];
      if (!in_place || (forks && t <= full)) a.table_out[(size_t)b * a.table_ld + t] = x;
    }
    if (threadIdx.x == 0) a.len_out[b] = forks ? n : a.seq_len[b];
  }
  if (!forks || rows == 0) return;
  const long long head = (long long)a.row_bytes << a.page_shift;  // bytes from one head to the next
  const long long at = (long long)blockIdx.z * a.layer_bytes + g0 * head;
  const uint8_t* const src = a.pages[kv] + (long long)page * a.page_bytes + at;
  uint8_t* const dst = a.pages[kv] + (long long)to * a.page_bytes + at;
  const int each = rows * (a.row_bytes / 16), all = heads * each;  // pieces of 16 bytes
  for (int e = threadIdx.x; e < all; e += 4 * 256) {
    u32x4 x[4];
    long long off[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int piece = min(e + k * 256, all - 1), g = piece / each;
      off[k] = g * head + (long long)(piece - g * each) * 16;
      x[k] = ld16(src + off[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (e + k * 256 < all) __builtin_nontemporal_store(x[k], reinterpret_cast<u32x4*>(dst + off[k]));
  }
  if (a.page_blocks) {
    const int used = (rows + kBlockRows - 1) / kBlockRows;
    const long long from = (long long)blockIdx.z * a.scale_layer + (long long)g0 * a.page_blocks;
    for (int k = threadIdx.x; k < heads * used; k += 256) {
      const long long x = from + k / used * a.page_blocks + k % used;
      a.scales[kv][x + (long long)to * a.scale_stride] = a.scales[kv][x + (long long)page * a.scale_stride];
    }
  }
}

int launch_fork(const char* who, const ooo_paged_batch* b, const Paged& p, ForkArgs& a, int n_layers,
                const int32_t* parent, const int32_t* fresh, int32_t* len_out, int32_t* table_out, void* stream) {
  OOO_REQUIRE(parent && fresh && len_out && table_out, OOO_ERR_INVALID, "%s: null pointer", who);
  OOO_REQUIRE((len_out == b->seq_len) == (table_out == b->page_table), OOO_ERR_INVALID,
              "%s: seq_len_out and table_out must both be the batch's, or neither", who);
  a.seq_len = p.seq_len;
  a.table = p.table;
  a.parent = parent;
  a.fresh = fresh;
  a.len_out = len_out;
  a.table_out = table_out;
  a.n_seqs = p.n_seqs;
  a.table_ld = p.table_ld;
  a.page_shift = p.page_shift;
  a.n_pages = p.n_pages;
  a.own_cap = p.own_cap;
  a.heads = p.Hkv;
  const long long head = (long long)a.row_bytes << p.page_shift;
  a.heads_each = (int)std::min<long long>(std::max<long long>(32768 / head, 1), p.Hkv);
  fork_kernel<<<dim3(2 * ((p.Hkv + a.heads_each - 1) / a.heads_each), p.n_seqs, n_layers), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ooo::ok();
}

}  // namespace
}  // namespace ooo

using namespace ooo;

extern "C" int ooo_paged_append8(const ooo_paged_batch* batch, const ooo_cache8* cache, int32_t layer,
                                 const void* qkv, int64_t qkv_ld, const void* q_norm, const void* k_norm, float eps,
                                 const int32_t* depth, double rope_theta, void* q_out, void* stream) {
  const char* const who = "ooo_paged_append8";
  AppendArgs a{};
  OOO_REQUIRE(cache, OOO_ERR_INVALID, "%s: cache is null", who);
  int rc = check_cache8(who, batch, cache, a.p, a.c);
  if (rc == OOO_OK) rc = take_layer(who, cache, layer, a.c);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(qkv && q_out, OOO_ERR_INVALID, "%s: null pointer", who);
  OOO_REQUIRE(rope_theta > 0.0 && eps >= 0.f, OOO_ERR_INVALID, "%s: rope_theta must be > 0, eps >= 0", who);
  const int D = batch->head_dim, per16 = batch->dt == OOO_BF16 ? 8 : 4;
  const long long width = (long long)(a.p.Hq + 2 * a.p.Hkv) * D;
  OOO_REQUIRE(qkv_ld >= width, OOO_ERR_INVALID, "%s: qkv_ld %lld below the row's %lld elements", who,
              (long long)qkv_ld, width);
  OOO_REQUIRE(qkv_ld % per16 == 0 && aligned16(qkv) && aligned16(q_out) && aligned16(q_norm) && aligned16(k_norm),
              OOO_ERR_UNSUPPORTED, "%s: a pointer or qkv_ld is not a multiple of 16 bytes", who);
  a.qkv = qkv;
  a.q_norm = q_norm;
  a.k_norm = k_norm;
  a.ld = qkv_ld;
  a.eps = eps;
  a.depth = depth;
  a.q_out = q_out;
  a.fr = rope_freq(rope_theta, D);
  a.span = a.p.n_rows / kSpan >= a.p.n_seqs ? kSpan : 1;
  const AppendGrid grid = append_grid(a);
  OOO_REQUIRE((grid.units + grid.rows) * 64 * kAppendWaves < (1ll << 32), OOO_ERR_UNSUPPORTED,
              "%s: n_rows %d needs more than 2^32 threads", who, a.p.n_rows);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (batch->dt == OOO_BF16 && D == 128) launch_append8<uint16_t, 128>(a, st);
  else if (batch->dt == OOO_BF16) launch_append8<uint16_t, 64>(a, st);
  else if (D == 128) launch_append8<float, 128>(a, st);
  else launch_append8<float, 64>(a, st);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ooo::ok();
}

extern "C" int ooo_paged_compact8(const ooo_paged_batch* batch, const ooo_cache8* cache, const int32_t* path,
                                  const int32_t* accept_len, int32_t path_cap, void* stream) {
  const char* const who = "ooo_paged_compact8";
  Paged p{};
  Cache8 c{};
  OOO_REQUIRE(cache, OOO_ERR_INVALID, "%s: cache is null", who);
  const int rc = check_cache8(who, batch, cache, p, c);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(path && accept_len, OOO_ERR_INVALID, "%s: null pointer", who);
  OOO_REQUIRE(path_cap >= 1, OOO_ERR_INVALID, "%s: path_cap must be >= 1", who);
  const dim3 grid((2 * p.Hkv + 3) / 4, p.n_seqs, cache->n_layers);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (batch->head_dim == 128)
    compact8_kernel<128><<<grid, 256, 0, st>>>(p, c, cache->layer_stride, cache->scale_layer_stride, path, accept_len,
                                               path_cap);
  else
    compact8_kernel<64><<<grid, 256, 0, st>>>(p, c, cache->layer_stride, cache->scale_layer_stride, path, accept_len,
                                              path_cap);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return ooo::ok();
}

extern "C" int ooo_paged_fork(const ooo_paged_batch* batch, void* k_pages, void* v_pages, int32_t n_layers,
                              int64_t layer_stride, const int32_t* parent, const int32_t* fresh,
                              int32_t* seq_len_out, int32_t* table_out, void* stream) {
  const char* const who = "ooo_paged_fork";
  Paged p{};
  const int rc = check_paged(who, batch, p);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(k_pages && v_pages, OOO_ERR_INVALID, "%s: null pointer", who);
  OOO_REQUIRE(n_layers >= 1, OOO_ERR_INVALID, "%s: n_layers must be >= 1", who);
  OOO_REQUIRE(n_layers == 1 || layer_stride >= 1, OOO_ERR_INVALID, "%s: layer_stride must be >= 1", who);
  OOO_REQUIRE(n_layers <= 65535, OOO_ERR_UNSUPPORTED, "%s: n_layers %d above 65535", who, n_layers);
  const int elt = batch->dt == OOO_BF16 ? 2 : 4;
  OOO_REQUIRE((n_layers == 1 || layer_stride * elt % 16 == 0) && aligned16(k_pages) && aligned16(v_pages),
              OOO_ERR_UNSUPPORTED, "%s: a pointer or layer_stride is not a multiple of 16 bytes", who);
  ForkArgs a{};
  a.pages[0] = (uint8_t*)k_pages;
  a.pages[1] = (uint8_t*)v_pages;
  a.page_bytes = p.page_stride * elt;
  a.layer_bytes = layer_stride * elt;
  a.row_bytes = batch->head_dim * elt;
  return launch_fork(who, batch, p, a, n_layers, parent, fresh, seq_len_out, table_out, stream);
}

extern "C" int ooo_paged_fork8(const ooo_paged_batch* batch, const ooo_cache8* cache, const int32_t* parent,
                               const int32_t* fresh, int32_t* seq_len_out, int32_t* table_out, void* stream) {
  const char* const who = "ooo_paged_fork8";
  Paged p{};
  Cache8 c{};
  OOO_REQUIRE(cache, OOO_ERR_INVALID, "%s: cache is null", who);
  const int rc = check_cache8(who, batch, cache, p, c);
  if (rc != OOO_OK) return rc;
  ForkArgs a{};
  for (int x = 0; x < 2; ++x) a.pages[x] = c.pages[x], a.scales[x] = c.scales[x];
  a.page_bytes = p.page_stride;
  a.layer_bytes = cache->layer_stride;
  a.row_bytes = batch->head_dim;
  a.scale_stride = c.scale_stride;
  a.scale_layer = cache->scale_layer_stride;
  a.page_blocks = c.page_blocks;
  return launch_fork(who, batch, p, a, cache->n_layers, parent, fresh, seq_len_out, table_out, stream);
}
