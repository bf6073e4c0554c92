// Attention with bf16 queries over one item of the plan where the pages hold
// 8-bit numbers (ooo_paged_attn8), on the matrix cores.
//
// The work, its items and the order of operands are those of paged_attn_bf16.h.
// A tile's rows are copied to LDS as they are, half the bytes, and become bf16
// on their way into a product: eight numbers of a key (or, for V^T, of a column:
// ds_read_b64_tr_b8 turns 8 x 16 of them) are eight bytes of a lane, and four
// v_cvt_scalef32_pk_bf16_fp8, which multiply by the block's power of two for
// nothing.  Both are exact, so scores and outputs are those of a bf16 cache with
// the same numbers.  (The 8-bit matrix product, with the queries split into two
// 8-bit numbers, would save K's conversion, but it adds the 32 products of a
// step aligned to the largest of them with some 14 bits: 2e-5 of the sum of
// their sizes is lost where float32 loses 1e-7.)
//
// What bounds it.  Wide tiles: the vector units, by softmax and conversions.
// Items of a wave alone: a CU's reads through the LDS DMA, which reaches 70 GB/s
// from L2 and 60 from HBM with 128 KiB on their way; 256 sequences of up to 4k
// own keys take 200 us (5.8 TB/s), and 73 where the same keys lie in L2.  Keys and
// values in registers, without LDS, took 233 and 97: a fragment of K is 16 rows
// of 64 bytes, which reach 51 GB/s.  Copies of the narrow and thin items are `nt`:
// a prompt that stays in the last cache takes less without it (8k for 64 rows 44
// us, not 54), keys read once more (256 rows over 32k and 4k own: 319, not 305).
#pragma once

#include "attn_tile.h"
#include "paged_attn_bf16.h"

namespace ooo {

// The LDS DMA of 4 bytes per lane from an address of the lane's own.
__device__ __forceinline__ void dma4_at(unsigned long long addr, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(addr) : "memory", "m0");
}
__device__ __forceinline__ void dma4_nt(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2 nt" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

// N (2 or 4) LDS DMA instructions of 16 bytes per lane, 1 KiB apart at both ends.
template <int N>
__device__ __forceinline__ void dma16s_nt(const void* base, const uint32_t (&voff)[N], uint32_t lds) {
  static_assert(N == 2 || N == 4, "a half-tile");
  if constexpr (N == 4)
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %5 nt\n\t"
        "global_load_lds_dwordx4 %2, %5 offset:%6 nt\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:%7 nt\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:%8 nt" ::"s"(lds),
        "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(base), "n"(1024), "n"(2 * 1024), "n"(3 * 1024)
        : "memory", "m0");
  else
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3 nt\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:1024 nt" ::"s"(lds),
        "v"(voff[0]), "v"(voff[1]), "s"(base)
        : "memory", "m0");
}

// LDS geometry of tiles of 8-bit rows: row-major, the 16-byte chunks of a row
// permuted so that no read meets itself in a bank.  A 16-byte read goes to the
// banks in groups of lanes 0-3, 12-15 and 20-27, of 4-11, 16-19 and 28-31, and the
// same 32 on: K's rows are then four quads of rows that differ in bits 2 and 3.
// The transpose reads of V are of 8 rows and two chunks, or of 16 rows and one.
// (With bit 4 of the row in the permutation too, every read of K took twice its
// time, by the count of conflicts.)
template <int D>
struct Ring8 {
  static constexpr int CH = D / 16;         // chunks of a row
  static constexpr int MAT = kTile * D;     // bytes of a tile of K or V
  static constexpr int HALF = 32 * D;       // of a half-tile, the rows of one scale
  static constexpr int BYTES = 128 * 1024;  // of the ring: 16 KiB a wave
  static constexpr int FOURTH = D / 2;      // what four rows on turn in an address
  static __device__ __forceinline__ int swz(int r, int c) {
    return c ^ (D == 128 ? (r & 6) | ((r >> 3) & 1) : ((r >> 1) & 2) | ((r >> 3) & 1));
  }
};

// Where the half-tiles that one wave copies and reads lie, and their scales.
// Step n is the 32 keys from k0 + n step on; lane l holds the address of step
// `base` + l.  Addresses are taken 64 steps at a time (turn), when the scales of
// those steps are asked for, and the page ids of the next 64; they go through
// LDS and have landed long before they are read: the waits for the tiles leave
// only the last requests on their way.
struct Window8 {
  static constexpr int BYTES = 6 * 256;  // of LDS a wave: page ids, then scales of K and of V, two of each
  const int32_t* ids;
  const uint8_t *ks, *vs;
  long long stride, head, scale_stride, scale_head;
  int k0, step, last, count, shift, n_pages, lane, row_bytes;
  uint8_t* buf;
  int base, kbase, vbase;
  uint32_t lo, hi, lds, kx, vx;
  bool bad;
  __device__ __forceinline__ int key(int n) const { return min(k0 + n * step, last); }
  __device__ __forceinline__ void start() {
    lds = __builtin_amdgcn_readfirstlane(lds_addr(buf));
    base = 0;
    kbase = vbase = -64;
    kx = vx = 0;
    bad = false;
    take(ids[key(lane) >> shift]);
    ask();
  }
  __device__ __forceinline__ uint32_t* word(int x, int n) const {
    return reinterpret_cast<uint32_t*>(buf + x * 512 + (n & 64) * 4) + lane;
  }
  __device__ __forceinline__ void take(int id) {
    const bool ok = id >= 0 && id < n_pages;
    bad = bad || __any(!ok);
    const long long page = ok ? id : 0;
    const int row = key(base + lane) & ((1 << shift) - 1);
    const unsigned long long at = (unsigned long long)(page * stride + head + (long long)(row & -32) * row_bytes);
    lo = (uint32_t)at;
    hi = (uint32_t)(at >> 32);
    // the words that the scales lie in
    const long long off = page * scale_stride + scale_head + row / kBlockRows;
    const unsigned long long k = (unsigned long long)(uintptr_t)(ks + off), v = (unsigned long long)(uintptr_t)(vs + off);
    *word(0, base) = (uint32_t)(8 * (k & 3) | 256 * 8 * (v & 3));
    dma4_at(k & ~3ull, lds + 512 + (base & 64) * 4);
    dma4_at(v & ~3ull, lds + 1024 + (base & 64) * 4);
  }
  __device__ __forceinline__ void ask() const {
    if (base + 64 >= count) return;
    dma4(ids, (uint32_t)(key(base + 64 + lane) >> shift) * 4u, lds + ((base + 64) & 64) * 4);
  }
  // Before at(n), for rising n.
  __device__ __forceinline__ void turn(int n) {
    if (n - base < 64) return;
    base += 64;
    take((int)*word(0, base));
    ask();
  }
  __device__ __forceinline__ long long at(int n) const {
    return (long long)((unsigned long long)(uint32_t)__builtin_amdgcn_readlane(hi, n - base) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane(lo, n - base));
  }
  // The scale of step n's keys or values, for rising n, behind the wait for step
  // n's keys.
  __device__ __forceinline__ float k_scale(int n) {
    if (n - kbase >= 64) {
      kbase += 64;
      kx = (*word(1, kbase) >> (*word(0, kbase) & 31) & 255) << 23;
    }
    return __uint_as_float(__builtin_amdgcn_readlane(kx, n & 63));
  }
  __device__ __forceinline__ float v_scale(int n) {
    if (n - vbase >= 64) {
      vbase += 64;
      vx = (*word(2, vbase) >> (*word(0, vbase) >> 8 & 31) & 255) << 23;
    }
    return __uint_as_float(__builtin_amdgcn_readlane(vx, n & 63));
  }
};

// Waits until only `ahead` (0 .. MOST) times PER and EXTRA requests are on their way.
template <int PER, int EXTRA, int MOST>
__device__ __forceinline__ void wait_ahead(int ahead) {
  if constexpr (MOST == 0) {
    wait_vmcnt<EXTRA>();
  } else {
    if (ahead >= MOST) wait_vmcnt<MOST * PER + EXTRA>();
    else wait_ahead<PER, EXTRA, MOST - 1>(ahead);
  }
}

// D = A(16x32) * B(32x16) + C with bf16 inputs and float32 accumulation.  Lane l
// holds A row (l % 16), k = 8*(l/16) .. +8; B column (l % 16), same k range; C/D
// element (row 4*(l/16) + r, column l % 16) in r.
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Eight numbers times a power of two.
__device__ __forceinline__ bf16x8 bf16_of(uint32_t lo, uint32_t hi, float up) {
  return as_bf16x8(u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, up, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, up, true)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, up, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, up, true))});
}

// As args_again.
__device__ __forceinline__ const PagedAttn8Args& args8_again() {
  return static_cast<const PagedAttn8Args&>(args_again());
}

// The steps of an item, 32 keys each, from key k0 on.
template <int D>
__device__ __forceinline__ Window8 window_of(const PagedAttn8Args& a, const Item& it, int g, int lane, int k0, int step,
                                             uint8_t* buf) {
  Window8 w;
  w.ids = it.flags & kShared ? a.p.shared_pages : a.p.table + (size_t)it.seq * a.p.table_ld;
  w.ks = a.c.scales[0];
  w.vs = a.c.scales[1];
  w.stride = a.p.page_stride;
  w.head = ((long long)g << a.p.page_shift) * D;
  w.scale_stride = a.c.scale_stride;
  w.scale_head = (long long)g * a.c.page_blocks;
  w.k0 = k0;
  w.step = step;
  w.last = it.limit - 1;
  w.count = it.t1 - it.t0;
  w.shift = a.p.page_shift;
  w.n_pages = a.p.n_pages;
  w.lane = lane;
  w.row_bytes = D;
  w.buf = buf;
  return w;
}

// The copies of a wave that works on half-tiles alone: its share of the ring is
// NS stages of a K half-tile and one of V.
template <int D>
struct HalfCopy {
  using R = Ring8<D>;
  static constexpr int HI = R::HALF / 1024;            // DMA instructions of a half-tile
  static constexpr int NS = 16384 / (2 * R::HALF);
  static constexpr int RPI = 1024 / D;                 // rows of an instruction
  uint32_t full[HI];
  int lane, keys;  // from the item's first on
  __device__ __forceinline__ HalfCopy(const Item& it, int ln) : lane(ln), keys(it.limit - 32 * it.t0) {
#pragma unroll
    for (int x = 0; x < HI; ++x) full[x] = off(x, 31) - 1024 * x;
  }
  // Instruction x: from the half-tile's first row to a lane's source; rows past
  // `last` repeat it.
  __device__ __forceinline__ uint32_t off(int x, int last) const {
    const int r = x * RPI + lane / R::CH;
    return (uint32_t)(min(r, last) * D + R::swz(r, lane % R::CH) * 16);
  }
  __device__ __forceinline__ void operator()(const uint8_t* src, int n, uint32_t to) const {
    const int last = keys - 32 * n - 1;
    if (last >= 31) {
      dma16s_nt<HI>(src, full, to);
    } else {
#pragma unroll
      for (int x = 0; x < HI; ++x) dma16_nt(src, off(x, max(last, 0)), to + x * 1024);
    }
  }
};

// One item by a workgroup (WIDE; every wave calls it) or by a wave alone.  PAST:
// its copies go past the caches.
template <int D, bool NEG, bool WIDE, bool PAST>
__device__ __forceinline__ void paged_attn8_item(int item, int g, int lane, int wave, uint8_t* ring,
                                                 uint64_t* mwords, uint8_t* windows, int* bad_s) {
  using R = Ring8<D>;
  constexpr int NW = kPagedWaves, RG = 4, NP = D / 8, DT = D / 32, S = D / 16;
  constexpr int V0 = 4 * R::MAT;       // of a wide ring: four stages of K, then of V
  constexpr int HI = HalfCopy<D>::HI, NS = HalfCopy<D>::NS;
  constexpr int kJoinMl = RG * NP * 64 * 16;  // where the joined halves' statistics lie, behind their sums
  static_assert(8 * R::MAT <= R::BYTES && kJoinMl + RG * 64 * 8 <= R::BYTES, "ring");
  const PagedAttn8Args& a = args8_again();
  const Paged p = a.p;
  const float scale = a.scale_log2e;
  const Item it = load_item(a.plan + (WIDE ? a.off_items_w : a.off_items_n), item);
  const int rg = WIDE ? wave % RG : 0, kh0 = WIDE ? wave / RG : 0;
  const int c = lane & 31, u = lane >> 5;
  const int qr = rg * 32 + c;                    // row of the block
  const bool on = qr < it.nq;
  const bool idle = rg * 32 >= it.nq;            // the whole group is past the block's rows
  const int qi = it.q0 + min(qr, it.nq - 1), i = qi / p.G, hq = g * p.G + qi - i * p.G;
  const long long row = (long long)it.row0 + i;
  // The queries: products 2 j and 2 j + 1 of a score take a key's 16 columns
  // 16 (2 j + u) on, as one read of K gives them.
  bf16x8 qf[S];
  {
    const uint16_t* qrow = (const uint16_t*)a.q + (row * p.Hq + hq) * D;
#pragma unroll
    for (int x = 0; x < S; ++x) qf[x] = as_bf16x8(ld16(qrow + 16 * (2 * (x / 2) + u) + 8 * (x & 1)));
  }
  Window8 window = window_of<D>(a, it, g, lane, WIDE ? kTileKeys * it.t0 + 32 * kh0 : 32 * it.t0,
                                WIDE ? kTileKeys : 32, windows + wave * Window8::BYTES);
  window.start();
  const int all = all_see(p, it);
  const uint8_t* const kp = (const uint8_t*)a.k;
  const uint8_t* const vp = (const uint8_t*)a.v;

  // LDS addresses of the fragments in the wave's first stage.  K read j: chunk
  // 2 j + u of row sigma(c), 32 j bytes away by the permutation's exclusive or.
  // V transpose read (16 keys kk, column block dt): row 16 kk + 8 (g16 / 2) +
  // li / 2, chunk 2 dt + g16 % 2, its half li % 2: 32 dt bytes away.
  const uint32_t k_lds = lds_addr(ring) + (WIDE ? kh0 * R::HALF : wave * 16384);
  const uint32_t v_lds = k_lds + (WIDE ? V0 : R::HALF);
  const int krow = sigma(c), g16 = lane >> 4, li = lane & 15;
  const int vrow = 8 * (g16 >> 1) + (li >> 1);
  uint32_t k_at = k_lds + krow * D + (R::swz(krow, u) << 4);
  uint32_t v_at = v_lds + vrow * D + (R::swz(vrow, g16 & 1) << 4) + 8 * (li & 1);

  // Ends the wait for the queries here: inside the loops it would be a wait for
  // the DMA in flight.  A negative scale (NEG) turns their signs, which is exact,
  // so that the largest score is the largest product and unseen keys stay at
  // -inf.
  auto queries_here = [&]() OOO_INLINE {
#pragma unroll
    for (int x = 0; x < S; ++x) asm volatile("" : "+v"(qf[x]));
    if constexpr (NEG) {
#pragma unroll
      for (int x = 0; x < S; ++x) qf[x] = as_bf16x8(__builtin_bit_cast(u32x4, qf[x]) ^ 0x80008000u);
    }
  };
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f;

  // ---- arithmetic of one half-tile (32 keys)
  auto kread1 = [&](int j) OOO_INLINE {
    return *(const u32x4 __attribute__((address_space(3)))*)(uintptr_t)(k_at ^ (32u * j));
  };
  auto kread = [&](u32x4 (&kr)[DT]) OOO_INLINE {
#pragma unroll
    for (int j = 0; j < DT; ++j) kr[j] = kread1(j);
  };
  auto score1 = [&](int x, const u32x4 (&kr)[DT], float up, const f32x16& acc) OOO_INLINE {
    return mfma32(bf16_of(kr[x / 2][2 * (x & 1)], kr[x / 2][2 * (x & 1) + 1], up), qf[x], acc);
  };
  auto scores = [&](const u32x4 (&kr)[DT], float up) OOO_INLINE {
    f32x16 acc = f32x16{};
#pragma unroll
    for (int x = 0; x < S; ++x) acc = score1(x, kr, up, acc);
    return acc;
  };
  auto vread = [&](int x) OOO_INLINE {  // 16 keys x / DT, column block x % DT
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                   (i32x2 __attribute__((address_space(3)))*)(uintptr_t)((v_at ^ (32u * (x % DT))) + 16 * (x / DT) * D)));
  };
  auto pv = [&](int x, const u32x2& v, float up, const bf16x8 (&pr)[2]) OOO_INLINE {
    oacc[x % DT] = mfma32(bf16_of(v[0], v[1], up), pr[x / DT], oacc[x % DT]);
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
    // A wave copies rows 8 wave .. 8 wave + 7 of every tile, which lie in its own
    // half: 1 KiB at head_dim 128 (16 bytes a lane), 512 bytes at 64 (4 bytes, twice).
    constexpr int PM = D == 128 ? 1 : 2;  // DMA instructions of a wave for K or V of a tile
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(ring) + wave * 8 * D);
    // from the half's first row in its page to a lane's source; rows past `last` repeat it
    auto rows_off = [&](int x, int last) OOO_INLINE -> uint32_t {
      if constexpr (D == 128) {
        const int r = 8 * wave + lane / 8;
        return (uint32_t)(min(r, last) & 31) * D + (uint32_t)R::swz(r, lane % 8) * 16u;
      } else {
        const int r = 8 * wave + 4 * x + lane / 16;
        return (uint32_t)(min(r, last) & 31) * D + (uint32_t)R::swz(r, lane % 16 / 4) * 16u + lane % 4 * 4u;
      }
    };
    auto copy1 = [&](const uint8_t* src, uint32_t off, uint32_t to, int x) OOO_INLINE {
      if constexpr (D == 128 && PAST) dma16_nt(src, off, to);
      else if constexpr (D == 128) dma16(src, off, to);
      else if constexpr (PAST) dma4_nt(src, off, to + x * 256);
      else dma4(src, off, to + x * 256);
    };
    uint32_t full_off[PM];
#pragma unroll
    for (int x = 0; x < PM; ++x) full_off[x] = rows_off(x, 63);
    auto stage = [&](int n) OOO_INLINE -> uint32_t { return (uint32_t)(n & 3) * R::MAT; };
    const int full = min(tiles, (it.limit >> 6) - it.t0);  // tiles whose keys all exist
    auto copy_full = [&](const uint8_t* src, uint32_t to, int x) OOO_INLINE {
      if (x < PM) copy1(src, full_off[x], to, x);
    };
    auto copy = [&](const uint8_t* src, int n, uint32_t to) OOO_INLINE {
      if (n < full) {
        copy_full(src, to, 0);
        copy_full(src, to, 1);
      } else if (n < tiles) {
#pragma unroll
        for (int x = 0; x < PM; ++x) copy1(src, rows_off(x, it.limit - kTileKeys * (it.t0 + n) - 1), to, x);
      }
    };
    // The order of copies, barriers and blocks is the bf16 kernel's.  Barrier m
    // says that K of tile m and V of tile m - 1 are here and that nobody reads K
    // of tile m - 1 or V of tile m - 3 any more.  Between it and the next, V of
    // tile m + 1 and K of tile m + 3 are asked for; where V lies is remembered
    // from K.
    long long src[3] = {0, 0, 0};  // of K of the three youngest tiles, the last one first
    auto aim = [&](int n) OOO_INLINE {
      src[2] = src[1];
      src[1] = src[0];
      src[0] = window.at(n);
    };
    auto ask_k = [&](int n) OOO_INLINE {
      if (n < tiles) window.turn(n);
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
      // tile n + 5.  Tiles whose keys all rows see and whose copies need no care go
      // through a body without conditions.
      u32x4 kr[DT];
      u32x2 vr[S];
      bf16x8 pf[2];
      kread(kr);
      ask_v(1, 1);
      ask_k(3);
      f32x16 sc = scores(kr, window.k_scale(0));
      barrier(1);
      k_at += to_next(0);
      kread(kr);
      bf16x8 kf[S];
      {
        const float up = window.k_scale(min(1, tiles - 1));
#pragma unroll
        for (int x = 0; x < S; ++x) kf[x] = bf16_of(kr[x / 2][2 * (x & 1)], kr[x / 2][2 * (x & 1) + 1], up);
      }
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
        const float k_up = window.k_scale(min(n + 2, tiles - 1)), v_up = window.v_scale(n);
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
          if (k < S) vr[k] = vread(k);
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
          pv(x, vr[x], v_up, pf);
          // K of tile n + 2: a read for two fragments, which follow two products later
          if (x % 2 == 0) kr[x / 2] = kread1(x / 2);
          if (x >= 2) kf[x - 2] = bf16_of(kr[x / 2 - 1][2 * (x & 1)], kr[x / 2 - 1][2 * (x & 1) + 1], k_up);
          if (PLAIN && x == S / 4) copy_full(kp + src[0], k_to, 0);
          if (PLAIN && x == S - S / 4) copy_full(kp + src[0], k_to, 1);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int x = S - 2; x < S; ++x)
          kf[x] = bf16_of(kr[x / 2][2 * (x & 1)], kr[x / 2][2 * (x & 1) + 1], k_up);
        sc = next;
      };
      for (int n = 0; n < tiles; ++n) {
        const int end = plain_end(tiles, (all >> 6) - it.t0, full, window.base + 64);
#pragma unroll 1
        for (; n < end; ++n) tile(Yes{}, n);
        if (n < tiles) tile(No{}, n);
      }
    }
  } else {
    // The wave's share of the ring: NS stages of a K half-tile and one of V.  A
    // half-tile is read into registers whole, K, then V, so that the one NS steps
    // on is asked for before the work on it begins.
    const uint32_t kd = __builtin_amdgcn_readfirstlane(k_lds);
    const HalfCopy<D> copy(it, lane);
    const int count = it.t1 - it.t0;
    const uint64_t* const words = p.mask + (size_t)row * p.W;
    queries_here();
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n < count) {
        copy(kp + window.at(n), n, kd + n * 2 * R::HALF);
        copy(vp + window.at(n), n, kd + n * 2 * R::HALF + R::HALF);
      }
    for (int n = 0; n < count; ++n) {
      const uint32_t st = kd + (uint32_t)(n % NS) * 2 * R::HALF;
      const int ahead = min(count - 1 - n, NS - 1);  // later half-tiles on their way, K and V
      const bool more = n + NS < count;
      u32x4 kr[DT];
      u32x2 vr[S];
      bf16x8 pf[2];
      wait_ahead<2 * HI, HI, NS - 1>(ahead);
      const float k_up = window.k_scale(n);
      kread(kr);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      long long src = 0;
      if (more) {
        window.turn(n + NS);
        src = window.at(n + NS);
        copy(kp + src, n + NS, st);
      }
      f32x16 sc = scores(kr, k_up);
      masked(sc, 32 * (it.t0 + n), words);
      settle(sc);
      weights(sc, new_max(row_max(sc, []() {})), pf, [](int) {});
      if (more) wait_vmcnt<(NS - 1) * 2 * HI + HI>();
      else wait_ahead<2 * HI, 0, NS - 1>(ahead);
      const float v_up = window.v_scale(n);
#pragma unroll
      for (int x = 0; x < S; ++x) vr[x] = vread(x);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy(vp + src, n + NS, st + R::HALF);
      const uint32_t step = n % NS == NS - 1 ? (uint32_t)(-2 * (NS - 1) * R::HALF) : (uint32_t)(2 * R::HALF);
      k_at += step;
      v_at += step;
#pragma unroll
      for (int x = 0; x < S; ++x) pv(x, vr[x], v_up, pf);
    }
  }
  bool bad = window.bad;

  const PagedAttn8Args& ea = args8_again();
  const Paged& ep = ea.p;
  const Item e = load_item(ea.plan + (WIDE ? ea.off_items_w : ea.off_items_n), item);
  const int eq = e.q0 + min(qr, e.nq - 1), ei = eq / ep.G;
  const long long row_e = (long long)e.row0 + ei;

  // A value of V that is not finite counts only for the rows that give its key
  // a weight, but the products multiply it by the zeros of the others, and
  // zero times it is NaN.  So a wave with a row of such sums adds its keys once
  // more, one by one, without those of weight zero.  A row whose weights are not
  // finite (its query, or a key that it sees) is NaN either way and no reason to.
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
          const int page = pages.at(t, bad), pr = t & ((1 << ep.page_shift) - 1);
          const long long base = (long long)page * ep.page_stride + (((long long)g << ep.page_shift) + pr) * D;
          const long long so = (long long)page * ea.c.scale_stride + (long long)g * ea.c.page_blocks + pr / kBlockRows;
          const float ku = scale_of(ea.c.scales[0] + so), vu = scale_of(ea.c.scales[1] + so);
          float s = 0.f;
#pragma unroll
          for (int y = 0; y < DT; ++y) {
            const u32x4 kk = ld16((const uint8_t*)ea.k + base + 16 * (2 * y + u));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const bf16x8 kb = bf16_of(kk[2 * h], kk[2 * h + 1], ku);
#pragma unroll
              for (int x = 0; x < 8; ++x) s = __builtin_fmaf((float)kb[x], (float)qf[2 * y + h][x], s);
            }
          }
          s += shfl_xor_f(s, 32);
          const float w = (bits >> j) & 1 ? __builtin_amdgcn_exp2f(fmaf(s, ea.scale_log2e, -m_use)) : 0.f;
          if (w == 0.f) continue;
          if (u == 0) l_run += w;
#pragma unroll
          for (int q = 0; q < NP; ++q) {
            float x[4];
            values4(*reinterpret_cast<const uint32_t*>((const uint8_t*)ea.v + base + 8 * q + 4 * u), vu, x);
            f32x16& o = oacc[q / 4];
#pragma unroll
            for (int y = 0; y < 4; ++y) o[4 * (q % 4) + y] += w * x[y];
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
      *reinterpret_cast<f32x2_t*>(ring + kJoinMl + (rg * 64 + lane) * 8) = f32x2_t{m_run, l_tot};
    }
    __syncthreads();
    if (kh0 == 1 || idle) return;
    const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(ring + kJoinMl + (rg * 64 + lane) * 8);
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

// One item of up to 16 query rows by a wave alone: decoding, where a sequence has
// one row for each query head of the group.  On 16x16x32 products it costs half
// the matrix and softmax work of the narrow item above, and it goes over 64 keys
// at a time, so that the chain of waits from K to P V is half as often: 256
// sequences take 201 us by either, by their reads, but 82 and 74 where the keys
// lie in L2, and beside the wide tiles of a 32k prompt 346 and 340.
// S^T = K Q^T in blocks of 16 keys, of which block t's row i is key 32 (t / 2) +
// 8 (i / 4) + 4 (t % 2) + i % 4, so that lane (c, u) holds row c's keys 8 u .. 8 u
// + 7 of either half in operand order; O^T = V^T P^T in blocks of 16 columns:
// columns 16 dt + 4 u + 0..3.
template <int D, bool NEG>
__device__ __forceinline__ void paged_attn8_thin(int item, int g, int lane, int wave, uint8_t* ring,
                                                 uint8_t* windows) {
  using R = Ring8<D>;
  constexpr int HI = HalfCopy<D>::HI, NS = HalfCopy<D>::NS / 2, S = D / 32, DT = D / 16;
  constexpr int ST = 4 * R::HALF;  // a stage: two half-tiles of K, two of V
  const PagedAttn8Args& a = args8_again();
  const Paged p = a.p;
  const float scale = a.scale_log2e;
  Item it = load_item(a.plan + a.off_items_n, item);
  it.limit = min(it.limit, 32 * it.t1);  // a last step may be half of one
  const int c = lane & 15, u = lane >> 4;
  const int qi = it.q0 + min(c, it.nq - 1), i = qi / p.G, hq = g * p.G + qi - i * p.G;
  const long long row = (long long)it.row0 + i;
  // products 2 j and 2 j + 1 take a key's 16 columns of chunk `part` + 2 j
  const int part = R::CH / 2 * (u & 1) + (u >> 1);
  bf16x8 qf[S];
  {
    const uint16_t* qrow = (const uint16_t*)a.q + (row * p.Hq + hq) * D;
#pragma unroll
    for (int x = 0; x < S; ++x) qf[x] = as_bf16x8(ld16(qrow + 16 * (part + 2 * (x / 2)) + 8 * (x & 1)));
  }
  Window8 window = window_of<D>(a, it, g, lane, 32 * it.t0, 32, windows + wave * Window8::BYTES);
  window.start();
  const int all = min(all_see(p, it), it.limit);
  const uint8_t* const kp = (const uint8_t*)a.k;
  const uint8_t* const vp = (const uint8_t*)a.v;
  const uint32_t kd = __builtin_amdgcn_readfirstlane(lds_addr(ring) + wave * 16384);
  const int krow = 8 * (c >> 2) + (c & 3), vrow = 8 * u + (c >> 1);
  uint32_t k_at = kd + krow * D + (R::swz(krow, part) << 4);
  uint32_t v_at = kd + 2 * R::HALF + vrow * D + (R::swz(vrow, 0) << 4) + 8 * (c & 1);
#pragma unroll
  for (int x = 0; x < S; ++x) asm volatile("" : "+v"(qf[x]));  // here, not inside the loop
  if constexpr (NEG) {
#pragma unroll
    for (int x = 0; x < S; ++x) qf[x] = as_bf16x8(__builtin_bit_cast(u32x4, qf[x]) ^ 0x80008000u);
  }
  f32x4 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  const HalfCopy<D> copy(it, lane);
  const int count = (it.t1 - it.t0 + 1) / 2;
  const uint64_t* const words = p.mask + (size_t)row * p.W;
#pragma unroll
  for (int n = 0; n < NS; ++n)
    if (n < count) {
      const long long s0 = window.at(2 * n), s1 = window.at(2 * n + 1);
      copy(kp + s0, 2 * n, kd + n * ST);
      copy(kp + s1, 2 * n + 1, kd + n * ST + R::HALF);
      copy(vp + s0, 2 * n, kd + n * ST + 2 * R::HALF);
      copy(vp + s1, 2 * n + 1, kd + n * ST + 3 * R::HALF);
    }
  for (int n = 0; n < count; ++n) {
    const uint32_t st = kd + (uint32_t)(n % NS) * ST;
    const int ahead = min(count - 1 - n, NS - 1);
    const bool more = n + NS < count;
    u32x4 kr[4][D / 64];
    u32x2 vr[2][DT];
    wait_ahead<4 * HI, 2 * HI, NS - 1>(ahead);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
        kr[t][j] = *(const u32x4 __attribute__((address_space(3)))*)(uintptr_t)((k_at ^ (32u * j) ^
                                                                                 (uint32_t)(R::FOURTH * (t & 1))) +
                                                                                (4 * (t & 1) + 32 * (t >> 1)) * D);
    const float k_up[2] = {window.k_scale(2 * n), window.k_scale(2 * n + 1)};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    long long src[2] = {0, 0};
    if (more) {
      window.turn(2 * (n + NS));
      src[0] = window.at(2 * (n + NS));
      src[1] = window.at(2 * (n + NS) + 1);
      copy(kp + src[0], 2 * (n + NS), st);
      copy(kp + src[1], 2 * (n + NS) + 1, st + R::HALF);
    }
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < S; ++x)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        s[t] = mfma16(bf16_of(kr[t][x / 2][2 * (x & 1)], kr[t][x / 2][2 * (x & 1) + 1], k_up[t >> 1]), qf[x], s[t]);
    const int lo = 32 * it.t0 + 64 * n;
    if (lo + 64 > all) {
      const uint64_t b = seen_in(p, it, i, words, lo) >> (8 * u);
      const uint32_t bits[2] = {(uint32_t)b, (uint32_t)(b >> 32)};
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (!((bits[j / 8] >> (j % 8)) & 1u)) s[j / 4][j % 4] = -INFINITY;
    }
    {  // as settle()
      const int x = __builtin_amdgcn_readfirstlane(__float_as_int(s[3][3]));
      asm volatile("" : "+v"(s[0]), "+v"(s[1]), "+v"(s[2]), "+v"(s[3]) : "s"(x));
    }
    float mt[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) mt[t] = max3f(s[t][0], s[t][1], s[t][2]);
    float mx = max3f(max3f(mt[0], s[0][3], mt[1]), max3f(s[1][3], mt[2], s[2][3]), max3f(mt[3], s[3][3], -INFINITY));
    {
      const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = max3f(__uint_as_float(h[0]), __uint_as_float(h[1]), -INFINITY);
      const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = max3f(__uint_as_float(q[0]), __uint_as_float(q[1]), -INFINITY) * scale;
    }
    // as in the narrow item: the reference maximum moves by 2^8 at a time
    if (__any(mx > m_run + 8.f)) {
      const float m_new = __builtin_fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    u32x4 pk[2];
    float ps[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[j / 2][2 * (j & 1)], scale, -m_use));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s[j / 2][2 * (j & 1) + 1], scale, -m_use));
      pk[j / 4][j % 4] = pack_bf16x2(e0, e1);
      ps[j & 1] = add_bf16x2(pk[j / 4][j % 4], ps[j & 1]);
    }
    l_run += ps[0] + ps[1];
    const bf16x8 pf[2] = {as_bf16x8(pk[0]), as_bf16x8(pk[1])};
    if (more) wait_vmcnt<(NS - 1) * 4 * HI + 2 * HI>();
    else wait_ahead<4 * HI, 0, NS - 1>(ahead);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        vr[h][dt] = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                       (i32x2 __attribute__((address_space(3)))*)(uintptr_t)((v_at ^ (16u * dt)) + h * R::HALF)));
    const float v_up[2] = {window.v_scale(2 * n), window.v_scale(2 * n + 1)};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) {
      copy(vp + src[0], 2 * (n + NS), st + 2 * R::HALF);
      copy(vp + src[1], 2 * (n + NS) + 1, st + 3 * R::HALF);
    }
    const uint32_t step = n % NS == NS - 1 ? (uint32_t)(-(NS - 1) * ST) : (uint32_t)ST;
    k_at += step;
    v_at += step;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        oacc[dt] = mfma16(bf16_of(vr[h][dt][0], vr[h][dt][1], v_up[h]), pf[h], oacc[dt]);
  }
  bool bad = window.bad;

  const PagedAttn8Args& ea = args8_again();
  const Paged& ep = ea.p;
  const Item e = load_item(ea.plan + ea.off_items_n, item);
  const int eq = e.q0 + min(c, e.nq - 1), ei = eq / ep.G;
  const long long row_e = (long long)e.row0 + ei;
  const auto whole = [](float x) { return (x + shfl_xor_f(x, 16)) + shfl_xor_f(x + shfl_xor_f(x, 16), 32); };

  // Sums that are not finite though the weights are: the keys once more, without
  // those of weight zero (paged_attn8_item).
  float z = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) z = __builtin_fmaf(oacc[dt][j], 0.f, z);
  bool again = __any(!(z == 0.f));
  if (again) again = __any(!(z == 0.f) && whole(l_run) < INFINITY);
  if (again) {
    const Pages pages(ep, e);
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int h = e.t0; h < e.t1; ++h) {
      const uint64_t bits = seen(ep, e, ei, (int)row_e, 32 * h);
#pragma unroll 1
      for (int j = 0; j < 32 && 32 * h + j < e.limit; ++j) {
        const int t = 32 * h + j;
        const int page = pages.at(t, bad), pr = t & ((1 << ep.page_shift) - 1);
        const long long base = (long long)page * ep.page_stride + (((long long)g << ep.page_shift) + pr) * D;
        const long long so = (long long)page * ea.c.scale_stride + (long long)g * ea.c.page_blocks + pr / kBlockRows;
        const float ku = scale_of(ea.c.scales[0] + so), vu = scale_of(ea.c.scales[1] + so);
        float s = 0.f;
#pragma unroll
        for (int y = 0; y < D / 64; ++y) {
          const u32x4 kk = ld16((const uint8_t*)ea.k + base + 16 * (part + 2 * y));
#pragma unroll
          for (int h2 = 0; h2 < 2; ++h2) {
            const bf16x8 kb = bf16_of(kk[2 * h2], kk[2 * h2 + 1], ku);
#pragma unroll
            for (int x = 0; x < 8; ++x) s = __builtin_fmaf((float)kb[x], (float)qf[2 * y + h2][x], s);
          }
        }
        s = whole(s);
        const float w = (bits >> j) & 1 ? __builtin_amdgcn_exp2f(fmaf(s, ea.scale_log2e, -m_use)) : 0.f;
        if (w == 0.f) continue;
        if (u == 0) l_run += w;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          float x[4];
          values4(*reinterpret_cast<const uint32_t*>((const uint8_t*)ea.v + base + 16 * dt + 4 * u), vu, x);
#pragma unroll
          for (int y = 0; y < 4; ++y) oacc[dt][y] += w * x[y];
        }
      }
    }
  }
  float l_tot = whole(l_run);
  const bool direct = e.flags & kDirect;
  if (c >= e.nq || (!direct && e.slot >= ea.max_slots)) return;
  if (bad) l_tot = __builtin_nanf("");
  if (direct) {
    const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;  // a row that sees no key is zero
    uint16_t* const orow = (uint16_t*)ea.out + (row_e * ep.Hq + g * ep.G + eq - ei * ep.G) * D + 4 * u;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<u32x2*>(orow + 16 * dt) = u32x2{pack_bf16x2(oacc[dt][0] * inv, oacc[dt][1] * inv),
                                                        pack_bf16x2(oacc[dt][2] * inv, oacc[dt][3] * inv)};
  } else {  // in the order of the narrow item's pieces
    const size_t sl = (size_t)e.slot * ep.Hkv + g;
    f32x4* const po = reinterpret_cast<f32x4*>(ea.part_o) + sl * (D / 8) * 64 + (u >> 1) * 64 + (u & 1) * 32 + c;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) po[2 * dt * 64] = oacc[dt];
    if (u == 0) reinterpret_cast<f32x2_t*>(ea.part_ml)[sl * 32 + c] = f32x2_t{m_run, l_tot};
  }
}

template <int D, bool NEG>
__global__ __launch_bounds__(64 * kPagedWaves) void paged_attn8_kernel(PagedAttn8Args) {
  __shared__ __attribute__((aligned(1024))) uint8_t ring[Ring8<D>::BYTES];
  __shared__ __attribute__((aligned(1024))) uint64_t mwords[4 * 32 * 16];
  __shared__ __attribute__((aligned(1024))) uint8_t windows[kPagedWaves * Window8::BYTES];
  __shared__ int bad_s;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int g, worker;
  {
    const PagedAttn8Args& a = args8_again();
    g = blockIdx.x % a.p.Hkv, worker = blockIdx.x / a.p.Hkv;
    const PlanHead head = load_head(a);
    if (!plan_fits(head, a.want)) return;
    // Tiles are read by every block of 128 query rows, so their copies keep them in
    // the caches: 8 tries over 4k 50.6 -> 49.9 us, 512 rows of a prompt over 16k 106
    // -> 102, 1175 over 4k 99 to 142, by the addresses, -> 89.  Beside many workers
    // that stream the sequences' own keys they do not: 256 rows over 32k (12 of 32
    // workers) take 300 us so and 306 else, 128 over 16k with 4 KV heads 84 and 87.
    // Twelve other shapes with prompts and own keys: within 4% either way, as repeats
    // of one form are.
    const bool past = 4 * head.narrow_workers > (int)gridDim.x / a.p.Hkv;
    each_wide(a, head, worker, [&](int item) OOO_INLINE {
      if (past) paged_attn8_item<D, NEG, true, true>(item, g, lane, wave, ring, mwords, windows, &bad_s);
      else paged_attn8_item<D, NEG, true, false>(item, g, lane, wave, ring, mwords, windows, &bad_s);
    });
  }
  const PagedAttn8Args& a = args8_again();
  const PlanHead head = load_head(a);
  const int narrow = worker - head.narrow_first;
  if (narrow < 0 || narrow >= head.narrow_workers) return;
  if (head.narrow_first == 0) __syncthreads();  // it may have done wide items
  const ScalarPtr fn = scalar_ptr(a.plan + a.off_first_n) + narrow * kPagedWaves + wave;
  const int n0 = fn[0], n1 = min(fn[1], a.max_items_n);
  for (int item = n0; item < n1; ++item) {
    if (load_item(a.plan + a.off_items_n, item).nq <= 16)
      paged_attn8_thin<D, NEG>(item, g, lane, wave, ring, windows);
    else
      paged_attn8_item<D, NEG, false, true>(item, g, lane, wave, ring, mwords, windows, &bad_s);
  }
}

}  // namespace ooo
