// Attention of a batch over a shared prompt and each sequence's own cache
// pages.  paged_plan.h says how the work is cut; here are the plan's kernels,
// the attention over one item and the join of the items' parts.
//
// For a query row, softmax(s q K^T) V over any split of its keys is joined
// from the parts' row maxima m, sums l = sum exp2(x - m) and unnormalised
// outputs O: O = sum_s exp2(m_s - m) O_s / sum_s exp2(m_s - m) l_s.  That is
// what lets the shared prompt be read once, for the stacked rows of all
// sequences, and long sequences be split.  Parts and statistics are float32.
#include "paged_attn_bf16.h"

namespace ooo {
namespace {

constexpr int kPlanThreads = 1024;

// ------------------------------------------------------------------- plan
// A sequence's rows and own tokens, bounded to what buffers and tables hold.
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
__device__ __forceinline__ int blocks_of(const PlanShape& s, int q) {
  return q <= s.narrow ? (q > 0) : (q + s.wide - 1) / s.wide;
}
// keys that query rows up to `last` (of the sequence) can see
__device__ __forceinline__ int keys_of(const Paged& p, const Seq& s, int last) {
  const int n = p.W ? min(s.rows, 64 * p.W) : last / p.G + 1;
  return min(s.len + n, p.own_cap);
}
struct Split {
  int tiles, per, n;
};
__device__ __forceinline__ Split split_of(long long tiles, int cost, long long budget) {
  const long long n = min(tiles, (tiles * cost + budget - 1) / budget);
  const long long per = n > 0 ? (tiles + n - 1) / n : 1;
  return Split{(int)tiles, (int)per, (int)((tiles + per - 1) / per)};
}

// Exclusive scan of two counts over the workgroup; the totals go to every thread.
__device__ __forceinline__ void scan2(long long& a, long long& b, long long& ta, long long& tb, long long (*sh)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long a0 = a, b0 = b;
  for (int off = 1; off < 64; off <<= 1) {
    const long long x = __shfl_up(a, off, 64), y = __shfl_up(b, off, 64);
    if (lane >= off) a += x, b += y;
  }
  __syncthreads();
  if (lane == 63) sh[wave][0] = a, sh[wave][1] = b;
  __syncthreads();
  long long pa = 0, pb = 0;
  ta = tb = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w == wave) pa = ta, pb = tb;
    ta += sh[w][0];
    tb += sh[w][1];
  }
  a += pa - a0;
  b += pb - b0;
}

// One workgroup.  First the total cost and the blocks' numbers, then the
// items and slots of every sequence behind those of the sequences before it.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(Paged p, PlanShape s, PlanHead head, uint8_t* plan) {
  __shared__ long long sh[kPlanThreads / 64][2];
  int4* const blocks = reinterpret_cast<int4*>(plan + s.off_blocks);
  int* const seq_block = reinterpret_cast<int*>(plan + s.off_seqs);
  Item* const items = reinterpret_cast<Item*>(plan + s.off_items);
  const int R = min(max(p.row_start[p.n_seqs], 0), p.n_rows);
  const int stack = R * p.G;  // query rows of a KV head

  long long cost = 0, nblk = 0;
  for (int b0 = 0; b0 < p.n_seqs; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    long long c = 0, n = 0;
    if (b < p.n_seqs) {
      const Seq q = seq_of(p, b, R);
      const int rows = q.rows * p.G;
      n = blocks_of(s, rows);
      const bool wide = rows > s.narrow;
      for (int j = 0; j < n; ++j) {
        const int last = wide ? min((j + 1) * s.wide, rows) - 1 : rows - 1;
        c += (long long)((keys_of(p, q, last) + kTileKeys - 1) / kTileKeys) * (wide ? s.cost_wide : s.cost_narrow);
      }
    }
    long long at = n, tc, tn;
    scan2(at, c, tn, tc, sh);
    if (b < p.n_seqs) seq_block[b] = (int)(nblk + at);
    cost += tc;
    nblk += tn;
  }
  const bool swide = stack > s.narrow;
  const int sblock = swide ? s.wide : s.narrow, scost = swide ? s.cost_wide : s.cost_narrow;
  const int sblocks = p.shared_len > 0 ? (stack + sblock - 1) / sblock : 0;
  const long long stiles = (p.shared_len + kTileKeys - 1) / kTileKeys;
  cost += sblocks * stiles * scost;
  const long long budget = max((cost + s.target - 1) / s.target, 1ll);
  const Split ss = split_of(sblocks ? stiles : 0, scost, budget);
  const int sgroups = sblock / s.group;
  if (threadIdx.x == 0) seq_block[p.n_seqs] = (int)nblk;

  // shared items: all row blocks of a run of tiles next to each other
  long long item0 = (long long)sblocks * ss.n, slot0 = item0 * sgroups;
  for (int k = threadIdx.x; k < item0; k += kPlanThreads) {
    const int sp = k / sblocks, blk = k - sp * sblocks;
    Item it{};
    it.flags = kShared | (swide ? kWide : 0);
    it.q0 = blk * sblock;
    it.nq = min(sblock, stack - it.q0);
    it.t0 = sp * ss.per;
    it.t1 = min(it.t0 + ss.per, ss.tiles);
    it.limit = it.len = p.shared_len;
    it.slot = (blk * ss.n + sp) * sgroups;
    if (k < s.max_items) items[k] = it;
  }
  for (int b0 = 0; b0 < p.n_seqs; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    long long ni = 0, ns = 0;
    Seq q{};
    int n = 0, rows = 0;
    if (b < p.n_seqs) {
      q = seq_of(p, b, R);
      rows = q.rows * p.G;
      n = blocks_of(s, rows);
    }
    const bool wide = rows > s.narrow;
    const int block = wide ? s.wide : s.narrow;
    const auto split = [&](int j, int& nq, int& limit) {
      nq = min(block, rows - j * block);
      limit = keys_of(p, q, j * block + nq - 1);
      return split_of((limit + kTileKeys - 1) / kTileKeys, wide ? s.cost_wide : s.cost_narrow, budget);
    };
    for (int j = 0; j < n; ++j) {
      int nq, limit;
      const Split sp = split(j, nq, limit);
      ni += sp.n;
      if (sblocks || sp.n > 1) ns += (long long)sp.n * ((nq + s.group - 1) / s.group);
    }
    long long ti, ts;
    scan2(ni, ns, ti, ts, sh);
    long long item = item0 + ni, slot = slot0 + ns;
    for (int j = 0; j < n; ++j) {
      int nq, limit;
      const Split sp = split(j, nq, limit);
      const bool direct = !sblocks && sp.n == 1;
      const int groups = (nq + s.group - 1) / s.group;
      const long long blk = seq_block[b] + j;
      if (blk < s.max_blocks) blocks[blk] = make_int4((int)slot, direct ? 0 : sp.n, groups, 0);
      for (int k = 0; k < sp.n; ++k, ++item) {
        Item it{};
        it.flags = (wide ? kWide : 0) | (direct ? kDirect : 0);
        it.seq = b;
        it.row0 = q.row0;
        it.q0 = j * block;
        it.nq = nq;
        it.t0 = k * sp.per;
        it.t1 = min(it.t0 + sp.per, sp.tiles);
        it.limit = limit;
        it.len = q.len;
        it.rows = q.rows;
        it.slot = (int)slot;
        if (!direct) slot += groups;
        if (item < s.max_items) items[item] = it;
      }
    }
    item0 += ti;
    slot0 += ts;
  }
  if (threadIdx.x == 0) {
    head.items = (int)min(item0, s.max_items);
    head.rows = R;
    head.shared_splits = sblocks ? ss.n : 0;
    head.shared_block = sblock;
    head.shared_slot0 = 0;
    *reinterpret_cast<PlanHead*>(plan) = head;
  }
}

// Where the parts of each query row lie.
__global__ __launch_bounds__(256) void plan_rows_kernel(Paged p, PlanShape s, uint8_t* plan) {
  const int x = blockIdx.x * 256 + threadIdx.x;
  const int R = min(max(p.row_start[p.n_seqs], 0), p.n_rows);
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
  RowSlots o{0, 0, 0, 0};
  if (at >= 0 && at < rows) {
    const int block = rows > s.narrow ? s.wide : s.narrow;
    const long long blk = reinterpret_cast<const int*>(plan + s.off_seqs)[lo] + at / block;
    if (blk < s.max_blocks) {
      const int4 d = reinterpret_cast<const int4*>(plan + s.off_blocks)[blk];
      const int in = at % block;
      o = RowSlots{d.x + in / s.group, d.y, d.z, in % s.group};
    }
  }
  reinterpret_cast<RowSlots*>(plan + s.off_rows)[x] = o;
}

// ------------------------------------------------------ attention, float32
__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// One item of up to 16 query rows on the f32 matrix instruction (16x16x4).
// The keys go in tiles of 16, dealt round-robin to the waves; a wave computes
// S^T = K Q^T and O^T += V^T P^T with its own online softmax, and the waves
// merge through LDS.  No operand is staged: K and V are read in runs of 4
// columns straight into operand registers, and P is already in B-operand
// order (lane (c, q) holds row c's scores of keys 4q .. 4q + 3).  Lane (c, q)
// of the O^T accumulator dt holds row c, columns 64 (dt / 4) + 16 q + 4 r +
// dt % 4.
template <int D>
__global__ __launch_bounds__(64 * 1024 / D) void paged_attn_f32_kernel(PagedAttnArgs a) {
  constexpr int NW = 1024 / D;
  constexpr int KS = D / 16;
  __shared__ f32x4 o_s[NW][KS][64];
  __shared__ f32x2_t ml_s[NW][16];
  __shared__ int odd_s[NW];
  const Paged& p = a.p;
  const int g = blockIdx.x % p.Hkv, item = blockIdx.x / p.Hkv;
  const PlanHead head = load_head(a);
  const Item it = load_item(a, item);  // within the plan's bound whatever it holds
  if (!plan_fits(head, a.want) || item >= head.items) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, qd = lane >> 4;
  const bool on = c < it.nq;
  const int qi = it.q0 + min(c, it.nq - 1), i = qi / p.G, head_q = g * p.G + qi - i * p.G;
  const long long row = (long long)it.row0 + i;
  const Pages pages(p, it);
  const int head_off = g << p.page_shift, in_page = (1 << p.page_shift) - 1;
  const float* const kp = (const float*)a.k;
  const float* const vp = (const float*)a.v;
  const int s0 = 4 * it.t0, s1 = min(4 * it.t1, (it.limit + 15) / 16);
  const int all = all_see(p, it);
  bool bad = false;

  f32x4 qv[KS], kv[KS];
  const float* const qrow = (const float*)a.q + (row * p.Hq + head_q) * D + 4 * qd;
#pragma unroll
  for (int s = 0; s < KS; ++s) qv[s] = load4(qrow + 16 * s) * a.scale_log2e;
  // rows past the keys re-read the last one (weight zero)
  const auto tile_base = [&](int t) {
    return (long long)pages.at(16 * t, bad) * p.page_stride + ((long long)head_off + ((16 * t) & in_page)) * D;
  };
  const auto load_k = [&](int t) {
    const float* kr = kp + tile_base(t) + (size_t)min(c, it.limit - 1 - 16 * t) * D + 4 * qd;
#pragma unroll
    for (int s = 0; s < KS; ++s) kv[s] = load4(kr + 16 * s);
  };
  f32x4 o[KS];
#pragma unroll
  for (int dt = 0; dt < KS; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  if (s0 + wave < s1) load_k(s0 + wave);
  for (int t = s0 + wave; t < s1; t += NW) {
    const int lo = 16 * t;
    f32x4 vv[4][D / 64];
    const float* const vb = vp + tile_base(t);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
        vv[r][h] = load4(vb + (size_t)min(4 * qd + r, it.limit - 1 - lo) * D + 64 * h + 4 * c);
    f32x4 score = {0.f, 0.f, 0.f, 0.f};
    // chains of eight products added in a tree: few roundings in a row
#pragma unroll
    for (int s = 0; s < KS; s += 4) {
      f32x4 sc[8];
#pragma unroll
      for (int ch = 0; ch < 8; ++ch) sc[ch] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) {
          const int x = s + ch / 2, e = 2 * (ch & 1) + j;
          sc[ch] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[x][e], qv[x][e], sc[ch], 0, 0, 0);
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
#pragma unroll
    for (int dt = 0; dt < KS; ++dt) {
      f32x4 pv[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int r = 0; r < 4; ++r)
        pv[r & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[r][dt >> 2][dt & 3], pr[r], pv[r & 1], 0, 0, 0);
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
  const int odd = __any(!((zero[0] + zero[1]) + (zero[2] + zero[3]) == 0.f));
  if (lane == 0) odd_s[wave] = (odd ? 1 : 0) | (__any(bad) ? 2 : 0);
  __syncthreads();
  float m = -INFINITY, den = 0.f;
  for (int w = 0; w < NW; ++w) m = fmaxf(m, ml_s[w][c][0]);
  const float base = m == -INFINITY ? 0.f : m;
  const bool poison = __any(lane < NW && (odd_s[lane < NW ? lane : 0] & 2));
  // A value of V that is not finite counts only for the query rows that give
  // its key a weight, but the matrix products multiply it by the zeros of the
  // others too, and zero times it is NaN.  So where a wave's sums are not
  // finite the block adds its keys once more, one by one and relative to the
  // rows' final exponents, without those of weight zero.
  if (__any(lane < NW && (odd_s[lane < NW ? lane : 0] & 1))) {
    __syncthreads();  // every wave has read ml_s and odd_s
    l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < KS; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t = s0 + wave; t < s1; t += NW) {
      const int lo = 16 * t;
      const long long tb = tile_base(t);
      const uint64_t mw = seen(p, it, i, (int)row, lo);
#pragma unroll 1
      for (int j = 0; j < 16 && lo + j < it.limit; ++j) {
        const float* kr = kp + tb + (size_t)j * D + 4 * qd;
        f32x4 s4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) s4 += load4(kr + 16 * s) * (load4(qrow + 16 * s) * a.scale_log2e);
        float sc = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        sc += shfl_xor_f(sc, 16);
        sc += shfl_xor_f(sc, 32);
        const float pk = (mw >> j) & 1ull ? exp2f(sc - base) : 0.f;
        if (pk == 0.f) continue;
        l_run += pk;
        const float* vr = vp + tb + (size_t)j * D + 16 * qd;
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x4 x = load4(vr + 64 * h + 4 * e);
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
  if (wave >= KS || !on) return;  // wave dt adds accumulator dt
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int w = 0; w < NW; ++w) {
    const f32x2_t ml = ml_s[w][c];
    const float wgt = exp2f(ml[0] - base);
    den += wgt * ml[1];
    acc += wgt * o_s[w][wave][lane];
  }
  if (poison) den = __builtin_nanf("");
  if (it.flags & kDirect) {
    const float inv = den == 0.f ? 0.f : 1.f / den;  // a row that sees no key is zero
    float* orow = (float*)a.out + (row * p.Hq + head_q) * D + 64 * (wave >> 2) + 16 * qd + (wave & 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) orow[4 * r] = acc[r] * inv;
  } else if (it.slot < a.max_slots) {
    const size_t sl = (size_t)it.slot * p.Hkv + g;
    reinterpret_cast<f32x4*>(a.part_o)[(sl * KS + wave) * 64 + lane] = acc;
    if (wave == 0 && qd == 0) reinterpret_cast<f32x2_t*>(a.part_ml)[sl * 16 + c] = f32x2_t{m, den};
  }
}

// ------------------------------------------------------------------- join
// One wave per (group of stacked query rows, KV head, accumulator piece): a
// lane joins 4 columns of one row over the row's shared and own slots.  Lane
// (c, q) of a piece holds row c and, in float32 (groups of 16), columns 64
// (piece / 4) + 16 q + 4 e + piece % 4; in bf16 (groups of 32) columns
// 8 piece + 4 q + e.
template <class T, int D>
__global__ __launch_bounds__(64) void join_kernel(PagedAttnArgs a) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int GR = BF ? 32 : 16, NP = D * GR / 256;
  const Paged& p = a.p;
  const PlanHead head = load_head(a);
  const int lane = threadIdx.x, c = lane % GR, qd = lane / GR;
  int w = blockIdx.x;
  const int pc = w % NP;
  w /= NP;
  const int g = w % p.Hkv, x = (w / p.Hkv) * GR + c;
  const int i = x / p.G, h = g * p.G + x - i * p.G;
  const bool fits = plan_fits(head, a.want);
  if (i >= (fits ? head.rows : min(p.row_start[p.n_seqs], p.n_rows))) return;
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
    put(f32x4{nan, nan, nan, nan});
    return;
  }
  const RowSlots rs = reinterpret_cast<const RowSlots*>(a.plan + a.off_rows)[x];
  if (rs.splits == 0) return;  // written by its item
  float m = -INFINITY, den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const auto add = [&](long long slot, int rw) {
    const size_t sl = (size_t)min(slot, a.max_slots - 1) * p.Hkv + g;
    const f32x2_t ml = reinterpret_cast<const f32x2_t*>(a.part_ml)[sl * GR + rw];
    const f32x4 o = reinterpret_cast<const f32x4*>(a.part_o)[(sl * NP + pc) * 64 + GR * qd + rw];
    const float mn = fmaxf(m, ml[0]), base = mn == -INFINITY ? 0.f : mn;
    const float wa = exp2f(m - base), wb = exp2f(ml[0] - base);
    den = den * wa + ml[1] * wb;
    acc = acc * wa;
    if (wb > 0.f) acc += o * wb;  // zero times an infinite sum is not zero
    m = mn;
  };
  const int sb = head.shared_block, sg = sb / GR;
  for (int s = 0; s < head.shared_splits; ++s)
    add(head.shared_slot0 + ((long long)(x / sb) * head.shared_splits + s) * sg + (x % sb) / GR, c);
  for (int s = 0; s < rs.splits; ++s) add(rs.slot + (long long)s * rs.stride, rs.row);
  put(acc * (den == 0.f ? 0.f : 1.f / den));
}

template <class T, int D>
void launch_attn(const PagedAttnArgs& a, const PlanShape& s, hipStream_t st) {
  const unsigned items = (unsigned)(s.max_items * a.p.Hkv);
  if constexpr (sizeof(T) == 2) paged_attn_bf16_kernel<D><<<items, 64 * kPagedWaves, 0, st>>>(a);
  else paged_attn_f32_kernel<D><<<items, 64 * 1024 / D, 0, st>>>(a);
  const long long groups = ((long long)a.p.n_rows * a.p.G + s.group - 1) / s.group;
  join_kernel<T, D><<<(unsigned)(groups * a.p.Hkv * (D * s.group / 256)), 64, 0, st>>>(a);
}

size_t workspace_bytes(const ooo_paged_batch& b, const PlanShape& s) {
  return (size_t)s.max_slots * b.n_kv_heads * s.group * (b.head_dim + 2) * sizeof(float);
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
  OOO_REQUIRE(plan, OOO_ERR_INVALID, "ooo_paged_plan: null pointer");
  OOO_REQUIRE(aligned16(plan), OOO_ERR_UNSUPPORTED, "ooo_paged_plan: plan is not 16-byte aligned");
  const PlanShape s = plan_shape(*batch);
  OOO_REQUIRE(plan_grid_ok(*batch, s), OOO_ERR_UNSUPPORTED, "ooo_paged_plan: more than 2^30 workgroups");
  OOO_REQUIRE(plan_bytes >= (size_t)s.bytes, OOO_ERR_CAPACITY, "ooo_paged_plan: plan of %lld bytes needed (got %zu)",
              s.bytes, plan_bytes);
  PlanHead head{};
  plan_key(*batch, head.key);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  plan_kernel<<<1, kPlanThreads, 0, st>>>(p, s, head, (uint8_t*)plan);
  const long long q = (long long)p.n_rows * p.G;
  plan_rows_kernel<<<(unsigned)((q + 255) / 256), 256, 0, st>>>(p, s, (uint8_t*)plan);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "ooo_paged_plan: launch failed: %s", hipGetErrorString(e));
  return ooo::ok();
}

extern "C" size_t ooo_paged_attn_workspace(const ooo_paged_batch* batch) {
  Paged p{};
  if (check_paged("ooo_paged_attn_workspace", batch, p) != OOO_OK) return 0;
  return workspace_bytes(*batch, plan_shape(*batch));
}

extern "C" int ooo_paged_attn(const ooo_paged_batch* batch, const void* plan, size_t plan_bytes, const void* q,
                              const void* k_pages, const void* v_pages, float scale, void* out, void* workspace,
                              size_t ws_bytes, void* stream) {
  PagedAttnArgs a{};
  const int rc = check_paged("ooo_paged_attn", batch, a.p);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(plan && q && k_pages && v_pages && out && workspace, OOO_ERR_INVALID, "ooo_paged_attn: null pointer");
  OOO_REQUIRE(aligned16(plan) && aligned16(q) && aligned16(k_pages) && aligned16(v_pages) && aligned16(out) &&
                  aligned16(workspace),
              OOO_ERR_UNSUPPORTED, "ooo_paged_attn: a pointer is not 16-byte aligned");
  const PlanShape s = plan_shape(*batch);
  OOO_REQUIRE(plan_grid_ok(*batch, s), OOO_ERR_UNSUPPORTED, "ooo_paged_attn: more than 2^30 workgroups");
  OOO_REQUIRE(plan_bytes >= (size_t)s.bytes, OOO_ERR_CAPACITY, "ooo_paged_attn: plan of %lld bytes needed (got %zu)",
              s.bytes, plan_bytes);
  const size_t need = workspace_bytes(*batch, s);
  OOO_REQUIRE(ws_bytes >= need, OOO_ERR_CAPACITY, "ooo_paged_attn: workspace of %zu bytes needed (got %zu)", need,
              ws_bytes);
  plan_key(*batch, a.want.key);
  a.plan = (const uint8_t*)plan;
  a.off_items = s.off_items;
  a.off_rows = s.off_rows;
  a.q = q;
  a.k = k_pages;
  a.v = v_pages;
  a.out = out;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + (size_t)s.max_slots * batch->n_kv_heads * s.group * batch->head_dim;
  a.max_slots = s.max_slots;
  a.scale_log2e = scale * 1.4426950408889634f;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool bf = batch->dt == OOO_BF16, wide = batch->head_dim == 128;
  if (bf && wide) launch_attn<uint16_t, 128>(a, s, st);
  else if (bf) launch_attn<uint16_t, 64>(a, s, st);
  else if (wide) launch_attn<float, 128>(a, s, st);
  else launch_attn<float, 64>(a, s, st);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "ooo_paged_attn: launch failed: %s", hipGetErrorString(e));
  return ooo::ok();
}
