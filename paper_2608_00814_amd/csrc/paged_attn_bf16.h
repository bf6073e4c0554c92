// bf16 attention over one item of the plan, on the matrix cores.
//
// Tiles, LDS layout and the order of operands are the tree attention's
// (tree_attn.hip): scores are computed transposed, S^T = K Q^T, and outputs as
// O^T = V^T P^T, so that with the rows of K permuted (sigma) a lane holds one
// query row: its softmax state, its probabilities, already in operand order,
// and half of its output columns (lane (c, u): row c of a group of 32, columns
// 8 n + 4 u + 0..3).
//
// A workgroup of eight waves works in one of two ways:
//  * wide, 33 to 128 query rows: four groups of 32 rows, two waves a group,
//    each with one 32-key half of every tile.  K and V tiles go through two
//    rings of four stages that all waves fill and read.  A SIMD holds one wave
//    of either half, and a tile costs them 1024 cycles of matrix products, about
//    1130 of vector work (512 of it exponentials) and 1070 of LDS traffic; at
//    two waves a SIMD (the accumulators leave no room for more) they overlap to
//    2100 cycles a tile, against 2650 with each wave's products, reads, copies
//    and vector work behind one another.
//  * narrow, up to 32 rows (a token or a small trie of one request): each wave
//    has items of its own, 1/8 of the LDS and no barrier, so that the start
//    and the end of one wave's items lie under the streams of the others.  A
//    half-tile's K is read into registers whole, so the next one's is on its
//    way while it is used, and V likewise: 16 KiB (head_dim 128) a wave.
//    Bound by HBM: one row of 256 sequences with 2049 keys each, 2.1 GB, in 326
//    us, 6.6 TB/s.  Beside the wide items of a 32k prompt a worker's waves 4 to 7,
//    the younger ones of their SIMDs, end at 282 us where waves 0 to 3, with as
//    many half-tiles, end at 217.
// Rows of a tile are copied by LDS DMA, 4 or 8 at a time, which never cross a
// page (pages hold a multiple of 16 rows).
#pragma once

#include "attn_tile.h"
#include "paged_attn.h"
#include "wide_schedule.h"

namespace ooo {

constexpr int kPagedWaves = 8;
struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

// The pages of an item as one wave reads them: lane l holds the byte offset of
// the KV head's rows in page index `base` + l, so that a tile's address takes
// no multiplication, and the next 64 ids are on their way to LDS (two buffers
// of 256 bytes).  Asked for a window ahead, at least 16 tiles, they have landed
// when the wave comes to them: it never waits for more than the last requests.
struct PageWindow {
  const int32_t* ids;
  int first, last, base, n_pages, lane;
  uint32_t lo, hi, lds;
  const uint8_t* buf;
  long long stride;   // bytes of a page
  long long head;     // bytes from a page's start to the head's rows
  bool bad;
  __device__ __forceinline__ PageWindow(const int32_t* p, int f, int l, int n, int ln, uint8_t* b, long long st,
                                        long long hd)
      : ids(p), first(f), last(l), base(0), n_pages(n), lane(ln), lds(__builtin_amdgcn_readfirstlane(lds_addr(b))),
        buf(b), stride(st), head(hd), bad(false) {
    take(ids[min(first + lane, last)]);
    ask();
  }
  __device__ __forceinline__ void take(int id) {
    const bool ok = id >= 0 && id < n_pages;
    bad = bad || __any(!ok);
    const unsigned long long at = (unsigned long long)(ok ? id : 0) * (unsigned long long)stride + (unsigned long long)head;
    lo = (uint32_t)at;
    hi = (uint32_t)(at >> 32);
  }
  __device__ __forceinline__ void ask() const {
    if (first + base + 64 > last) return;
    dma4(ids, (uint32_t)min(first + base + 64 + lane, last) * 4u, lds + ((base + 64) & 64) * 4);
  }
  // Before the pages of a tile or half-tile whose first key lies on page
  // `index`; they never straddle two windows (64 is a multiple of their pages).
  __device__ __forceinline__ void turn(int index) {
    if (index - first - base < 64) return;
    base += 64;
    take(*reinterpret_cast<const int*>(buf + (base & 64) * 4 + lane * 4));
    ask();
  }
  __device__ __forceinline__ long long at(int index) const {
    const int x = index - first - base;
    return (long long)((unsigned long long)(uint32_t)__builtin_amdgcn_readlane(hi, x) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane(lo, x));
  }
};

// The kernel's arguments and the item once more, from memory: what the ends of
// an item need would otherwise stay in registers through its loop, which has
// none to spare.
__device__ __forceinline__ const PagedAttnArgs& args_again() {
  typedef const __attribute__((address_space(4))) PagedAttnArgs* Ptr;
  Ptr p = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const PagedAttnArgs*)p;
}

// One item by a workgroup (WIDE; every wave calls it) or by a wave alone.
template <int D, bool NEG, bool WIDE>
__device__ __forceinline__ void paged_attn_item(int item, int g, int lane, int wave,
                                                uint8_t* ring, uint64_t* mwords, uint8_t* windows, int* bad_s) {
  using R = KvRing<D>;
  constexpr int NW = kPagedWaves, RG = 4, NP = D / 8;
  constexpr int PM = R::DMA_MAT / NW;  // DMA instructions per wave and matrix of a tile
  constexpr int HB = 32 * R::ROWB;     // bytes of a half-tile of K or V
  constexpr int HI = HB / 1024;        // its DMA instructions
  constexpr int V0 = 4 * R::MAT;
  const PagedAttnArgs& a = args_again();
  const Paged p = a.p;
  const float scale = a.scale_log2e;
  const Item it = load_item(a.plan + (WIDE ? a.off_items_w : a.off_items_n), item);
  constexpr int kKeys = WIDE ? kTileKeys : kTileKeys / 2;
  const int32_t* const ids = it.flags & kShared ? p.shared_pages : p.table + (size_t)it.seq * p.table_ld;
  const int rg = WIDE ? wave % RG : 0, kh0 = WIDE ? wave / RG : 0;
  const int c = lane & 31, u = lane >> 5;
  const int qr = rg * 32 + c;                    // row of the block
  const bool on = qr < it.nq;
  const bool idle = rg * 32 >= it.nq;            // the whole group is past the block's rows
  const int qi = it.q0 + min(qr, it.nq - 1), i = qi / p.G, hq = g * p.G + qi - i * p.G;
  const long long row = (long long)it.row0 + i;
  // the queries and the page ids are on their way together
  bf16x8 qf[D / 16];
  {
    const uint16_t* qrow = (const uint16_t*)a.q + (row * p.Hq + hq) * D;
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) qf[dk] = as_bf16x8(ld16(qrow + 16 * dk + 8 * u));
  }
  PageWindow window(ids, kKeys * it.t0 >> p.page_shift, (min(kKeys * it.t1, it.limit) - 1) >> p.page_shift,
                    p.n_pages, lane, windows + wave * 512, 2 * p.page_stride,
                    ((long long)g << p.page_shift) * R::ROWB);
  const int all = all_see(p, it);
  const int in_page = (1 << p.page_shift) - 1;
  const uint8_t* const kp = (const uint8_t*)a.k;
  const uint8_t* const vp = (const uint8_t*)a.v;

  // LDS addresses of the fragments, from one of K's and one of V's each, in the
  // wave's first stage (offsets of a read reach 64 KiB, so K and V stages have
  // bases of their own).  K fragment (k-step dk): logical chunk 2 dk + u of row
  // sigma(c), 32 dk bytes away by the permutation's exclusive or.  V^T
  // transpose-read source (column block dt, half h): row 4 h + 8 (g16 / 2) +
  // li / 4 of 16, columns 32 dt + 16 (g16 % 2) + 4 (li % 4) .. + 3: 64 dt bytes
  // away, and h turns the permutation's bit of row 4.
  const uint32_t k_lds = lds_addr(ring) + (WIDE ? 32 * kh0 * R::ROWB : wave * R::MAT);
  const uint32_t v_lds = WIDE ? k_lds + V0 : k_lds + HB;
  const int krow = sigma(c), g16 = lane >> 4, li = lane & 15;
  const int vrow = 8 * (g16 >> 1) + (li >> 2), vcol = 16 * (g16 & 1) + 4 * (li & 3);
  uint32_t k_at = k_lds + krow * R::ROWB + (R::swz(krow, u) << 4);
  uint32_t v_at = v_lds + vrow * R::ROWB + (R::swz(vrow, vcol >> 3) << 4) + (vcol & 7) * 2;
  constexpr uint32_t kRow4 = D == 128 ? 16 : 64;

  // Ends the wait for the queries here: inside the loops it would be a wait for
  // the DMA in flight.  A negative scale (NEG) turns their signs, which is exact,
  // so that the largest score is the largest product and unseen keys stay at
  // -inf.  (Asked here instead of by a kernel of its own: 0.3 to 0.7 us a call.)
  auto queries_here = [&]() OOO_INLINE {
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) asm volatile("" : "+v"(qf[dk]));
    if constexpr (NEG) {
#pragma unroll
      for (int dk = 0; dk < D / 16; ++dk)
        qf[dk] = as_bf16x8(__builtin_bit_cast(u32x4, qf[dk]) ^ 0x80008000u);
    }
  };
  f32x16 oacc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f;

  // ---- arithmetic of one half-tile (32 keys): as in the tree attention
  auto kfrag = [&](int dk) OOO_INLINE {
    return as_bf16x8(*(const u32x4 __attribute__((address_space(3)))*)(uintptr_t)(k_at ^ (32u * dk)));
  };
  auto kread = [&](bf16x8 (&kf)[D / 16]) OOO_INLINE {
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) kf[dk] = kfrag(dk);
  };
  auto scores = [&](const bf16x8 (&kf)[D / 16]) OOO_INLINE {
    f32x16 acc = f32x16{};
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) acc = mfma32(kf[dk], qf[dk], acc);
    return acc;
  };
  auto vfrag = [&](int x) OOO_INLINE {  // 16 keys x / (D / 32), column block x % (D / 32)
    constexpr int DT = D / 32;
    u32x2 lohi[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      lohi[h] = __builtin_bit_cast(
          u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                     (i16x4 __attribute__((address_space(3)))*)(uintptr_t)((v_at ^ (64u * (x % DT)) ^ (kRow4 * h)) +
                                                                           (16 * (x / DT) + 4 * h) * R::ROWB)));
    return as_bf16x8(u32x4{lohi[0][0], lohi[0][1], lohi[1][0], lohi[1][1]});
  };
  auto pv = [&](int x, const bf16x8& v, const bf16x8 (&pr)[2]) OOO_INLINE {
    constexpr int DT = D / 32;
    oacc[x % DT] = mfma32(v, pr[x / DT], oacc[x % DT]);
  };
  auto row_max = [&](const f32x16& s, auto between) OOO_INLINE {
    float m0 = max3f(s[0], s[1], s[2]), m1 = max3f(s[8], s[9], s[10]);
    m0 = max3f(m0, s[3], s[4]);
    m1 = max3f(m1, s[11], s[12]);
    between();
    m0 = max3f(m0, s[5], s[6]);
    m1 = max3f(m1, s[13], s[14]);
    const float mx = max3f(max3f(m0, s[7], m1), s[15], -INFINITY);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    return max3f(__uint_as_float(sw[0]), __uint_as_float(sw[1]), -INFINITY) * scale;
  };
  auto masked = [&](f32x16& s, int lo, const uint64_t* words) OOO_INLINE {
    if (lo + 32 > all) {
      // lane value j is key 16 (j / 8) + 8 u + j % 8
      const uint32_t b = (uint32_t)seen_in(p, it, i, words, lo) >> (8 * u);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (!((b >> (16 * (j / 8) + j % 8)) & 1u)) s[j] = -INFINITY;
    }
  };
  // The reference maximum moves only when some row grows by more than 2^8, so
  // probabilities stay <= 256 and O, l are rescaled rarely.
  auto new_max = [&](float mx) OOO_INLINE {
    if (__any(mx > m_run + 8.f)) {
      const float m_new = __builtin_fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) oacc[dt] *= alpha;
      m_run = m_new;
    }
    return m_run == -INFINITY ? 0.f : m_run;
  };
  // Probabilities, two at a time, each pair behind the next pair's exponents;
  // between(k) goes with pair k.  They go into the product rounded to bf16, the
  // matrix cores' operand, and the rounded ones into the sum: the weights that
  // multiply V then sum to one, and the rounding (half a step, 2^-8, each)
  // moves an output by that share of sum p |v - out| alone.
  auto weights = [&](const f32x16& s, float m_use, bf16x8 (&pf)[2], auto between) OOO_INLINE {
    float x[2] = {fmaf(s[0], scale, -m_use), fmaf(s[1], scale, -m_use)};
    float pr[2][2], ps[2] = {0.f, 0.f};
    u32x4 pk[2];
#pragma unroll
    for (int k = 0; k <= 8; ++k) {
      if (k < 8) between(k);
      if (k < 8) {
        pr[k & 1][0] = __builtin_amdgcn_exp2f(x[0]);
        pr[k & 1][1] = __builtin_amdgcn_exp2f(x[1]);
        asm volatile("" : "+v"(pr[k & 1][0]), "+v"(pr[k & 1][1]));  // not later
      }
      if (k < 7) {
        x[0] = fmaf(s[2 * k + 2], scale, -m_use);
        x[1] = fmaf(s[2 * k + 3], scale, -m_use);
      }
      if (k > 0) {
        const float* e = pr[(k - 1) & 1];
        pk[(k - 1) / 4][(k - 1) % 4] = pack_bf16x2(e[0], e[1]);
        ps[k & 1] = add_bf16x2(pk[(k - 1) / 4][(k - 1) % 4], ps[k & 1]);
      }
    }
    pf[0] = as_bf16x8(pk[0]);
    pf[1] = as_bf16x8(pk[1]);
    l_run += ps[0] + ps[1];
  };
  // A DMA instruction copies rows [r0, r0 + RPI) of a tile or half-tile at keys
  // lo on, of which n exist (rows past those repeat the last).  rows_at:
  // bytes from the pool's start to the first of them; rows_off: bytes from
  // there to a lane's source, the same for all r0 equal modulo 16 while every
  // row exists.
  auto rows_at = [&](int lo, int n, int r0) OOO_INLINE {
    const int key = lo + min(r0, n - 1);
    return window.at(key >> p.page_shift) + (key & in_page) * R::ROWB;
  };
  auto rows_off = [&](int n, int r0) OOO_INLINE -> uint32_t {
    const int r = r0 + lane / R::CH;
    return (uint32_t)(min(r, n - 1) - min(r0, n - 1)) * R::ROWB + (uint32_t)R::swz(r, lane % R::CH) * 16u;
  };

  if constexpr (WIDE) {
    if (threadIdx.x == 0) *bad_s = 0;
    const int tiles = it.t1 - it.t0;
    // mask words of the block's rows, for the tiles that hold new rows
    if (p.W && !(it.flags & kShared) && kTileKeys * it.t1 > it.len) {
      const int n = RG * 32 * 2 * p.W / 64;
      for (int j = wave; j < n; j += NW) {
        const int e = j * 64 + lane, r = e / (2 * p.W), k = e - r * (2 * p.W);
        const int node = (it.q0 + min(r, it.nq - 1)) / p.G;
        dma4(p.mask, (uint32_t)((it.row0 + node) * 2 * p.W + k) * 4u, lds_addr(mwords) + j * 256);
      }
    }
    const uint64_t* const words = mwords + qr * p.W;
    // A wave copies rows 8 wave .. 8 wave + 7 of every tile: one page.
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(ring) + wave * 8 * R::ROWB);
    uint32_t full_off[PM];
#pragma unroll
    for (int x = 0; x < PM; ++x) full_off[x] = rows_off(kTileKeys, wave * 8 + x * R::RPI);
    auto stage = [&](int n) OOO_INLINE -> uint32_t { return (uint32_t)(n & 3) * R::MAT; };
    const int full = min(tiles, (it.limit >> 6) - it.t0);  // tiles whose keys all exist
    // Instruction x of K or V of tile n.
    auto copy_full = [&](const uint8_t* src, uint32_t to, int x) OOO_INLINE {
      if (x == 0) dma16_nt(src, full_off[0], to);
      else if (x < PM) dma16_nt_at<1024>(src, full_off[PM - 1], to);
    };
    auto copy = [&](const uint8_t* src, int n, uint32_t to) OOO_INLINE {
      if (n < full) {
        copy_full(src, to, 0);
        copy_full(src, to, 1);
      } else if (n < tiles) {
        const int last = it.limit - kTileKeys * (it.t0 + n) - 1, r0 = min(wave * 8, last);
#pragma unroll
        for (int x = 0; x < PM; ++x) {
          const int r = wave * 8 + x * R::RPI + lane / R::CH;
          dma16_nt(src, (uint32_t)(min(r, last) - r0) * R::ROWB + (uint32_t)R::swz(r, lane % R::CH) * 16u,
                   to + x * 1024);
        }
      }
    };
    // Barrier m says that K of tile m and V of tile m - 1 are here and that
    // nobody reads K of tile m - 1 or V of tile m - 3 any more.  Between it and
    // the next, V of tile m + 1 and K of tile m + 3 are asked for; where V lies
    // is remembered from K.
    long long src[3] = {0, 0, 0};  // of K of the three youngest tiles, the last one first
    auto aim = [&](int n) OOO_INLINE {
      src[2] = src[1];
      src[1] = src[0];
      const int lo = kTileKeys * (it.t0 + n);
      src[0] = rows_at(lo, it.limit - lo, wave * 8);
    };
    auto ask_k = [&](int n) OOO_INLINE {
      if (n < tiles) window.turn(kTileKeys * (it.t0 + n) >> p.page_shift);
      aim(min(n, tiles - 1));
      copy(kp + src[0], n, dst + stage(n));
    };
    auto ask_v = [&](int n, int back) OOO_INLINE { copy(vp + src[back], n, dst + V0 + stage(n)); };
    auto barrier = [&](int m) OOO_INLINE {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (copies_left(m, tiles) == 2) wait_vmcnt<2 * PM>();
      else if (copies_left(m, tiles) == 1) wait_vmcnt<PM>();
      else wait_vmcnt<0>();
      wg_barrier();
    };
    auto to_next = [&](int n) OOO_INLINE -> uint32_t {  // from the stage of tile n to that of n + 1
      return (n & 3) == 3 ? (uint32_t)(-3 * R::MAT) : (uint32_t)R::MAT;
    };
    queries_here();
    ask_k(0);
    ask_k(1);
    ask_v(0, 1);
    ask_k(2);
    barrier(0);
    if (idle) {  // copies and keeps step
#pragma unroll 1
      for (int m = 1; m <= tiles + 1; ++m) {
        ask_v(m, 1);
        ask_k(m + 2);
        barrier(m);
      }
    } else {
      // A tile is a block of vector work, the softmax of tile n, with the
      // products of the scores of tile n + 1 and the reads of V of tile n between,
      // and one of the products P V of tile n with the reads of K of tile n + 2
      // between.  Wave A (kh0 = 0) has its barrier between the two, wave B before
      // the first, so that the blocks of the two alternate on a SIMD.  The first
      // block asks for V, of tile n + 2 by A and n + 3 by B, the second for K of
      // tile n + 5.  A wave issues in order, a vector instruction in five cycles
      // and a scalar one that needs the last's result in eight, so what goes to
      // one pipe is spread over the block, and tiles whose keys all rows see and
      // whose copies need no care go through a body without conditions (2100
      // cycles; 2580 with them).
      constexpr int S = D / 16;  // products of a block
      bf16x8 kf[S], vv[S], pf[2];
      kread(kf);
      ask_v(1, 1);
      ask_k(3);
      f32x16 sc = scores(kf);
      barrier(1);
      k_at += to_next(0);
      kread(kf);
      if (kh0 == 1) ask_v(2, 1);
      ask_k(4);
      auto tile = [&](auto plain, int n) OOO_INLINE {
        constexpr bool PLAIN = decltype(plain)::value;
        auto turn = [&]() OOO_INLINE {
          if constexpr (PLAIN) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wait_vmcnt<2 * PM>();
            wg_barrier();
          } else {
            barrier(n + 2);
          }
        };
        if (kh0 == 1) turn();
        f32x16 next = mfma32(kf[0], qf[0], f32x16{});
        const int nv = n + 2 + kh0;
        const uint8_t* const v_src = vp + (kh0 == 0 ? src[2] : src[1]);
        const uint32_t v_to = dst + V0 + stage(nv);
        if constexpr (!PLAIN) {
          masked(sc, kTileKeys * (it.t0 + n) + 32 * kh0, words);
          copy(v_src, nv, v_to);
        }
        settle(sc);
        const float m_use = new_max(row_max(sc, [&]() OOO_INLINE {
          __builtin_amdgcn_sched_barrier(0);
          next = mfma32(kf[1], qf[1], next);
          __builtin_amdgcn_sched_barrier(0);
        }));
        weights(sc, m_use, pf, [&](int k) OOO_INLINE {
          if (k + 2 < S) next = mfma32(kf[k + 2], qf[k + 2], next);
          if (k < S) vv[k] = vfrag(k);
          if (PLAIN && k == 2) copy_full(v_src, v_to, 0);
          if (PLAIN && k == 5) copy_full(v_src, v_to, 1);
          __builtin_amdgcn_sched_barrier(0);
        });
        v_at += to_next(n);
        // else the compiler moves them to their use, behind wave A's barrier
        asm volatile("" : "+v"(pf[0]), "+v"(pf[1]), "+v"(l_run));
        if (kh0 == 0) turn();
        k_at += to_next(n + 1);
        if constexpr (PLAIN) aim(min(n + 5, tiles - 1));  // the last one again where there is none
        else ask_k(n + 5);
        const uint32_t k_to = dst + stage(n + 5);
#pragma unroll
        for (int x = 0; x < S; ++x) {
          pv(x, vv[x], pf);
          kf[x] = kfrag(x);
          if (PLAIN && x == S / 4) copy_full(kp + src[0], k_to, 0);
          if (PLAIN && x == S - S / 4) copy_full(kp + src[0], k_to, 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        sc = next;
      };
      for (int n = 0; n < tiles; ++n) {
        const int wt = (int)min((long long)tiles,
                                ((long long)(window.first + window.base + 64) << p.page_shift >> 6) - it.t0);
        const int end = plain_end(tiles, (all >> 6) - it.t0, full, wt);
#pragma unroll 1
        for (; n < end; ++n) tile(Yes{}, n);
        if (n < tiles) tile(No{}, n);
      }
    }
  } else {
    // the wave's share of the ring: a K half-tile, then one of V
    const uint32_t kd = __builtin_amdgcn_readfirstlane(k_lds), vd = kd + HB;
    constexpr int H2 = HI / 2;  // instructions of 16 rows, which lie on one page
    uint32_t full_off[H2];
#pragma unroll
    for (int x = 0; x < H2; ++x) full_off[x] = rows_off(32, x * R::RPI);
    long long at[2];  // from the pool's start to the asked half-tile's rows 0 and 16
    auto aim = [&](int h) OOO_INLINE {
      window.turn(32 * h >> p.page_shift);
#pragma unroll
      for (int x = 0; x < 2; ++x) at[x] = rows_at(32 * h, it.limit - 32 * h, 16 * x);
    };
    auto ask = [&](const uint8_t* pool, int h, uint32_t dst) OOO_INLINE {
      const int n = it.limit - 32 * h;
      if (n >= 32) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          dma16_nt(pool + at[y], full_off[0], dst + y * H2 * 1024);
          dma16_nt_at<1024>(pool + at[y], full_off[1], dst + y * H2 * 1024);
          if constexpr (H2 == 4) {
            dma16_nt_at<2 * 1024>(pool + at[y], full_off[2], dst + y * H2 * 1024);
            dma16_nt_at<3 * 1024>(pool + at[y], full_off[3], dst + y * H2 * 1024);
          }
        }
      } else {
#pragma unroll 1
        for (int x = 0; x < HI; ++x)
          dma16_nt(pool + rows_at(32 * h, n, x * R::RPI), rows_off(n, x * R::RPI), dst + x * 1024);
      }
    };
    const uint64_t* const words = p.mask + (size_t)row * p.W;
    int h = it.t0;
    const int h1 = it.t1;
    queries_here();
    aim(h);
    ask(kp, h, kd);
    ask(vp, h, vd);
    for (; h < h1; ++h) {
      const bool more = h + 1 < h1;
      bf16x8 kf[D / 16], vv[D / 16], pf[2];
      wait_vmcnt<HI>();  // K is here, V on its way
      kread(kf);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) {
        aim(h + 1);
        ask(kp, h + 1, kd);
      }
      f32x16 sc = scores(kf);
      masked(sc, 32 * h, words);
      settle(sc);
      weights(sc, new_max(row_max(sc, []() {})), pf, [](int) {});
      if (more) wait_vmcnt<HI>();
      else wait_vmcnt<0>();
#pragma unroll
      for (int x = 0; x < D / 16; ++x) vv[x] = vfrag(x);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) ask(vp, h + 1, vd);
#pragma unroll
      for (int x = 0; x < D / 16; ++x) pv(x, vv[x], pf);
    }
  }
  bool bad = window.bad;

  const PagedAttnArgs& ea = args_again();
  const Paged& ep = ea.p;
  const Item e = load_item(ea.plan + (WIDE ? ea.off_items_w : ea.off_items_n), item);
  const int eq = e.q0 + min(qr, e.nq - 1), ei = eq / ep.G;
  const long long row_e = (long long)e.row0 + ei;

  // A value of V that is not finite counts only for the rows that give its key
  // a weight, but the products multiply it by the zeros of the others, and
  // zero times it is NaN.  So a wave with a row of such sums adds its keys once
  // more, one by one, without those of weight zero.  A row whose weights are not
  // finite (its query, or a key that it sees) is NaN either way and no reason
  // to: 64 rows over a 4k prompt took 1600 us, not 41, for one NaN query.
  if (!idle) {
    float z = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 16; ++j) z = __builtin_fmaf(oacc[dt][j], 0.f, z);
    bool again = __any(!(z == 0.f));
    if (again) again = __any(!(z == 0.f) && l_run + shfl_xor_f(l_run, 32) < INFINITY);
    if (again) {
      const Pages pages(ep, e);
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      l_run = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = f32x16{};
      const int step = WIDE ? 2 : 1, h1 = WIDE ? 2 * e.t1 : e.t1;
      for (int h = WIDE ? 2 * e.t0 + kh0 : e.t0; h < h1 && 32 * h < e.limit; h += step) {
        const uint64_t bits = seen(ep, e, ei, (int)row_e, 32 * h);
#pragma unroll 1
        for (int j = 0; j < 32 && 32 * h + j < e.limit; ++j) {
          const int t = 32 * h + j;
          const long long base = (long long)pages.at(t, bad) * ep.page_stride +
                                 (((long long)g << ep.page_shift) + (t & ((1 << ep.page_shift) - 1))) * D;
          float s = 0.f;
#pragma unroll
          for (int dk = 0; dk < D / 16; ++dk) {
            const bf16x8 kk = as_bf16x8(ld16((const uint16_t*)ea.k + base + 16 * dk + 8 * u));
#pragma unroll
            for (int x = 0; x < 8; ++x) s = __builtin_fmaf((float)kk[x], (float)qf[dk][x], s);
          }
          s += shfl_xor_f(s, 32);
          const float w = (bits >> j) & 1 ? __builtin_amdgcn_exp2f(fmaf(s, ea.scale_log2e, -m_use)) : 0.f;
          if (w == 0.f) continue;
          if (u == 0) l_run += w;
#pragma unroll
          for (int q = 0; q < NP; ++q) {
            const u32x2 x = *reinterpret_cast<const u32x2*>((const uint16_t*)ea.v + base + 8 * q + 4 * u);
            f32x16& o = oacc[q / 4];
            o[4 * (q % 4)] += w * __uint_as_float(x[0] << 16);
            o[4 * (q % 4) + 1] += w * __uint_as_float(x[0] & 0xFFFF0000u);
            o[4 * (q % 4) + 2] += w * __uint_as_float(x[1] << 16);
            o[4 * (q % 4) + 3] += w * __uint_as_float(x[1] & 0xFFFF0000u);
          }
        }
      }
    }
  }

  float l_tot = l_run + shfl_xor_f(l_run, 32);
  if constexpr (WIDE) {
    if (__any(bad)) *bad_s = 1;
    wait_vmcnt<0>();
    __syncthreads();  // the ring is free, bad_s complete
  }
  auto piece = [&](int q) OOO_INLINE {
    return f32x4{oacc[q / 4][4 * (q % 4)], oacc[q / 4][4 * (q % 4) + 1], oacc[q / 4][4 * (q % 4) + 2],
                 oacc[q / 4][4 * (q % 4) + 3]};
  };
  uint16_t* const orow = (uint16_t*)ea.out + (row_e * ep.Hq + g * ep.G + eq - ei * ep.G) * D + 4 * u;
  auto put = [&](int q, f32x4 o, float inv) OOO_INLINE {
    u32x2 pk;
    pk[0] = pack_bf16x2(o[0] * inv, o[1] * inv);
    pk[1] = pack_bf16x2(o[2] * inv, o[3] * inv);
    *reinterpret_cast<u32x2*>(orow + 8 * q) = pk;
  };
  const bool direct = e.flags & kDirect;
  const size_t sl = (size_t)(e.slot + rg) * ep.Hkv + g;
  f32x4* const po = reinterpret_cast<f32x4*>(ea.part_o) + sl * NP * 64 + lane;
  f32x2_t* const pml = reinterpret_cast<f32x2_t*>(ea.part_ml) + sl * 32 + c;
  if (!direct && e.slot + (e.nq + 31) / 32 > ea.max_slots) return;
  if constexpr (WIDE) {
    // join the two key halves of each row group through the ring
    if (kh0 == 1 && !idle) {
#pragma unroll
      for (int q = 0; q < NP; ++q)
        *reinterpret_cast<f32x4*>(ring + ((rg * NP + q) * 64 + lane) * 16) = piece(q);
      *reinterpret_cast<f32x2_t*>(ring + V0 + (rg * 64 + lane) * 8) = f32x2_t{m_run, l_tot};
    }
    __syncthreads();
    if (kh0 == 1 || idle) return;
    const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(ring + V0 + (rg * 64 + lane) * 8);
    const float mn = __builtin_fmaxf(m_run, ml[0]), base = mn == -INFINITY ? 0.f : mn;
    const float a0 = __builtin_amdgcn_exp2f(m_run - base), a1 = __builtin_amdgcn_exp2f(ml[0] - base);
    l_tot = l_tot * a0 + ml[1] * a1;
    if (*bad_s) l_tot = __builtin_nanf("");
    const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;  // a row that sees no key is zero
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const f32x4 o1 = *reinterpret_cast<const f32x4*>(ring + ((rg * NP + q) * 64 + lane) * 16);
      f32x4 o = piece(q) * a0;
      if (a1 > 0.f) o += o1 * a1;
      if (direct) {
        if (on) put(q, o, inv);
      } else {
        po[q * 64] = o;
      }
    }
    if (!direct && u == 0) *pml = f32x2_t{mn, l_tot};
  } else if (on) {
    if (bad) l_tot = __builtin_nanf("");
    const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      if (direct) put(q, piece(q), inv);
      else po[q * 64] = piece(q);
    }
    if (!direct && u == 0) *pml = f32x2_t{m_run, l_tot};
  }
}

template <int D, bool NEG>
__global__ __launch_bounds__(64 * kPagedWaves) void paged_attn_bf16_kernel(PagedAttnArgs) {
  __shared__ __attribute__((aligned(1024))) uint8_t ring[8 * KvRing<D>::MAT];  // four stages of K, then of V
  __shared__ __attribute__((aligned(1024))) uint64_t mwords[4 * 32 * 16];
  __shared__ __attribute__((aligned(1024))) uint8_t windows[kPagedWaves * 512];
  __shared__ int bad_s;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int g, worker;
  {
    const PagedAttnArgs& a = args_again();
    g = blockIdx.x % a.p.Hkv, worker = blockIdx.x / a.p.Hkv;
    const PlanHead head = load_head(a);
    if (!plan_fits(head, a.want)) return;
    each_wide(a, head, worker, [&](int item) OOO_INLINE {
      paged_attn_item<D, NEG, true>(item, g, lane, wave, ring, mwords, windows, &bad_s);
    });
  }
  const PagedAttnArgs& a = args_again();
  const PlanHead head = load_head(a);
  const int narrow = worker - head.narrow_first;
  if (narrow < 0 || narrow >= head.narrow_workers) return;
  if (head.narrow_first == 0) __syncthreads();  // it may have done wide items
  const ScalarPtr fn = scalar_ptr(a.plan + a.off_first_n) + narrow * kPagedWaves + wave;
  const int n0 = fn[0], n1 = min(fn[1], a.max_items_n);
  for (int item = n0; item < n1; ++item)
    paged_attn_item<D, NEG, false>(item, g, lane, wave, ring, mwords, windows, &bad_s);
}

}  // namespace ooo
