// bf16 attention over one item of the plan, on the matrix cores.
//
// Tiles, LDS layout and the order of operands are the tree attention's
// (tree_attn.hip): scores are computed transposed, S^T = K Q^T, and outputs as
// O^T = V^T P^T, so that with the rows of K permuted (sigma) a lane holds one
// query row: its softmax state, its probabilities, already in operand order,
// and half of its output columns (lane (c, u): row c of a group of 32, columns
// 8 n + 4 u + 0..3).
//
// A workgroup of eight waves takes its item in one of two ways:
//  * wide, 33 to 128 query rows: four groups of 32 rows, two waves a group,
//    each with one 32-key half of every tile.  K and V tiles go through a ring
//    of four stages that all waves fill and read.  The two waves of a group
//    run half a tile apart, one in its matrix products while the other is in
//    its softmax.  Bound by the matrix cores: a tile is 2.1 MFLOP a wave.
//  * narrow, up to 32 rows (a token or a small trie of one request): each wave
//    takes every eighth 32-key half-tile for all rows, with 1/8 of the LDS to
//    itself and no barrier.  K is read into registers whole, so the next
//    half-tile's K is on its way while this one's is used, and V likewise:
//    32 KiB (head_dim 128) ahead of each pair of waves.  Bound by HBM.
// Rows of a tile are copied by LDS DMA, 4 or 8 at a time, which never cross a
// page (pages hold a multiple of 16 rows); a page's id is fetched a tile ahead.
#pragma once

#include <type_traits>

#include "attn_tile.h"
#include "paged_attn.h"

namespace ooo {

constexpr int kPagedWaves = 8;

template <int D>
__global__ __launch_bounds__(64 * kPagedWaves) void paged_attn_bf16_kernel(PagedAttnArgs a) {
  using R = KvRing<D>;
  constexpr int NW = kPagedWaves, RG = 4, NP = D / 8;
  constexpr int PM = R::DMA_MAT / NW;  // DMA instructions per wave and matrix of a tile
  constexpr int PER = 2 * PM;
  constexpr int HB = 32 * R::ROWB;     // bytes of a half-tile of K or V
  constexpr int HI = HB / 1024;        // its DMA instructions
  __shared__ __attribute__((aligned(1024))) uint8_t ring[8 * R::MAT];  // four stages of K, then of V
  __shared__ __attribute__((aligned(1024))) uint64_t mwords[RG * 32 * 16];
  __shared__ int bad_s;
  constexpr int V0 = 4 * R::MAT;

  const Paged& p = a.p;
  const int g = blockIdx.x % p.Hkv, item = blockIdx.x / p.Hkv;
  const PlanHead head = load_head(a);
  const Item it = load_item(a, item);  // within the plan's bound whatever it holds
  if (!plan_fits(head, a.want) || item >= head.items) return;
  const Pages pages(p, it);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool wide = it.flags & kWide;
  const int rg = wide ? wave % RG : 0, kh0 = wide ? wave / RG : 0;
  const int c = lane & 31, u = lane >> 5;
  const int qr = rg * 32 + c;                    // row of the block
  const bool on = qr < it.nq;
  const bool idle = rg * 32 >= it.nq;            // the whole group is past the block's rows
  const int qi = it.q0 + min(qr, it.nq - 1), i = qi / p.G, hq = g * p.G + qi - i * p.G;
  const long long row = (long long)it.row0 + i;
  const int all = all_see(p, it);
  const int in_page = (1 << p.page_shift) - 1;
  const uint16_t* const kp = (const uint16_t*)a.k;
  const uint16_t* const vp = (const uint16_t*)a.v;
  bool bad = false;
  if (threadIdx.x == 0) bad_s = 0;

  // K fragment (k-step dk): logical chunk 2 dk + u of row sigma(c).  V^T
  // transpose-read source (column block dt, half h): row 4 h + 8 (g16 / 2) +
  // li / 4 of 16, columns 32 dt + 16 (g16 % 2) + 4 (li % 4) .. + 3.
  const int krow = sigma(c);
  uint32_t koff[D / 16];
#pragma unroll
  for (int dk = 0; dk < D / 16; ++dk) koff[dk] = (krow + 32 * kh0) * R::ROWB + (R::swz(krow, 2 * dk + u) << 4);
  const int g16 = lane >> 4, li = lane & 15;
  uint32_t voff[D / 32][2];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int vr = 4 * h + 8 * (g16 >> 1) + (li >> 2);
      const int col = 32 * dt + 16 * (g16 & 1) + 4 * (li & 3);
      voff[dt][h] = (vr + 32 * kh0) * R::ROWB + (R::swz(vr, col >> 3) << 4) + (col & 7) * 2;
    }

  bf16x8 qf[D / 16];
  {
    const uint16_t* qrow = (const uint16_t*)a.q + (row * p.Hq + hq) * D;
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) qf[dk] = as_bf16x8(ld16(qrow + 16 * dk + 8 * u));
  }
  // Ends the wait for the queries here: inside the loops it would be a wait for
  // the DMA in flight.
  auto queries_here = [&]() OOO_INLINE {
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) asm volatile("" : "+v"(qf[dk]));
  };
  f32x16 oacc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f;

  auto page_base = [&](int id, int row_in) OOO_INLINE {  // elements from the pool's start
    return (long long)id * p.page_stride + (((long long)g << p.page_shift) + row_in) * D;
  };
  // ---- arithmetic of one half-tile (32 keys): as in the tree attention
  auto kread = [&](const uint8_t* ks, bf16x8 (&kf)[D / 16]) OOO_INLINE {
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) kf[dk] = as_bf16x8(*reinterpret_cast<const u32x4*>(ks + koff[dk]));
  };
  auto scores = [&](const bf16x8 (&kf)[D / 16]) OOO_INLINE {
    f32x16 acc = f32x16{};
#pragma unroll
    for (int dk = 0; dk < D / 16; ++dk) acc = mfma32(kf[dk], qf[dk], acc);
    return acc;
  };
  auto vread = [&](const uint8_t* vs, int ks, bf16x8 (&vv)[D / 32]) OOO_INLINE {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      u32x2 lohi[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* q = vs + voff[dt][h] + ks * 16 * R::ROWB;
        lohi[h] = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((i16x4 __attribute__((address_space(3)))*)OOO_LDS(q)));
      }
      vv[dt] = as_bf16x8(u32x4{lohi[0][0], lohi[0][1], lohi[1][0], lohi[1][1]});
    }
  };
  auto pv = [&](const bf16x8 (&vv)[D / 32], const bf16x8& pr) OOO_INLINE {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = mfma32(vv[dt], pr, oacc[dt]);
  };
  auto row_max = [&](const f32x16& s) OOO_INLINE {
    float m0 = max3f(s[0], s[1], s[2]), m1 = max3f(s[8], s[9], s[10]);
    m0 = max3f(m0, s[3], s[4]);
    m1 = max3f(m1, s[11], s[12]);
    m0 = max3f(m0, s[5], s[6]);
    m1 = max3f(m1, s[13], s[14]);
    const float mx = max3f(max3f(m0, s[7], m1), s[15], -INFINITY);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    return max3f(__uint_as_float(sw[0]), __uint_as_float(sw[1]), -INFINITY) * a.scale_log2e;
  };
  // The reference maximum moves only when some row grows by more than 2^8, so
  // probabilities stay <= 256 and O, l are rescaled rarely.  Probabilities go
  // into the product rounded to bf16, the matrix cores' operand.
  auto softmax = [&](f32x16& s, uint32_t bits, bf16x8 (&pf)[2]) OOO_INLINE {
    if (__any(bits != ~0u)) {
      // lane value j is key 16 (j / 8) + 8 u + j % 8
      const uint32_t b = bits >> (8 * u);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (!((b >> (16 * (j / 8) + j % 8)) & 1u)) s[j] = -INFINITY;
    }
    const float mx = row_max(s);
    if (__any(mx > m_run + 8.f)) {
      const float m_new = __builtin_fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) oacc[dt] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      float pr[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pr[e] = __builtin_amdgcn_exp2f(fmaf(s[8 * k2 + e], a.scale_log2e, -m_use));
        ps[e % 4] += pr[e];
      }
      u32x4 pk;
#pragma unroll
      for (int e = 0; e < 4; ++e) pk[e] = pack_bf16x2(pr[2 * e], pr[2 * e + 1]);
      pf[k2] = as_bf16x8(pk);
    }
    l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
  };
  // DMA of the rows [r0, r0 + RPI) of the keys from lo on (n of them exist;
  // rows past those repeat the last) from the page `id` that holds the first
  auto copy_rows = [&](const uint16_t* pool, int id, int lo, int n, int r0, uint32_t dst) OOO_INLINE {
    const int rb = min(r0, n - 1), r = r0 + lane / R::CH;
    const uint32_t off = (uint32_t)(min(r, n - 1) - rb) * R::ROWB + (uint32_t)R::swz(r, lane % R::CH) * 16u;
    dma16_nt(pool + page_base(id, (lo + rb) & in_page), off, dst);
  };

  if (wide) {
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
    // A wave copies rows RPI (8 i + wave) of every tile (i < PM).
    int ids[PM];
    auto fetch = [&](int t) OOO_INLINE {
#pragma unroll
      for (int x = 0; x < PM; ++x)
        ids[x] = pages.at(min(kTileKeys * t + (x * NW + wave) * R::RPI, it.limit - 1), bad);
    };
    auto issue = [&](int t, auto stage_c) OOO_INLINE {
      constexpr int ST = decltype(stage_c)::value;
      const int lo = kTileKeys * t, n = it.limit - lo;
      const uint32_t kl = lds_addr(ring) + ST * R::MAT + wave * 1024, vl = lds_addr(ring) + V0 + ST * R::MAT + wave * 1024;
#pragma unroll
      for (int x = 0; x < PM; ++x) copy_rows(kp, ids[x], lo, n, (x * NW + wave) * R::RPI, kl + x * NW * 1024);
#pragma unroll
      for (int x = 0; x < PM; ++x) copy_rows(vp, ids[x], lo, n, (x * NW + wave) * R::RPI, vl + x * NW * 1024);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    fetch(it.t0);
    issue(it.t0, I0{});
    if (tiles > 1) fetch(it.t0 + 1);
    wait_vmcnt<0>();
    queries_here();
    __syncthreads();
    if (tiles > 1) {
      issue(it.t0 + 1, I1{});
      if (tiles > 2) fetch(it.t0 + 2);
    }
    if (tiles > 2) {
      issue(it.t0 + 2, I2{});
      if (tiles > 3) fetch(it.t0 + 3);
    }
    auto tile_bits = [&](int t) OOO_INLINE -> uint32_t {  // of the wave's half
      const int lo = kTileKeys * t + 32 * kh0;
      if (lo + 32 <= all) return ~0u;
      return (uint32_t)seen_in(p, it, i, mwords + qr * p.W, lo);
    };
    auto pv_tile = [&](auto stage_c, const bf16x8 (&pf)[2]) OOO_INLINE {
      constexpr int ST = decltype(stage_c)::value;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        bf16x8 vv[D / 32];
        vread(ring + V0 + ST * R::MAT, ks, vv);
        pv(vv, pf[ks]);
      }
    };
    // Wave A (kh0 = 0) runs the scores and the softmax of tile i between
    // barriers i and i + 1, wave B (kh0 = 1) the softmax of tile i - 1, its
    // product with V and the scores of tile i: their matrix and vector blocks
    // alternate on a SIMD.  Because tile i - 1 is read after barrier i, tile
    // i + 2 is requested behind that barrier, into the stage of tile i - 2.
    bf16x8 pf_hold[2];
    f32x16 sc_hold;
    auto body = [&](auto role_c, int n, auto st_c) OOO_INLINE {
      constexpr bool B = decltype(role_c)::value;
      constexpr int ST = decltype(st_c)::value;
      if (n > 0) {
        wait_tiles<PER, 1>(min(1, tiles - 1 - n));
        wg_barrier();
        if (!idle) {
          if constexpr (B) softmax(sc_hold, tile_bits(it.t0 + n - 1), pf_hold);
          __builtin_amdgcn_sched_barrier(0);
          pv_tile(std::integral_constant<int, (ST + 3) % 4>{}, pf_hold);
        }
      }
      f32x16 sc;
      if (!idle) {
        bf16x8 kf[D / 16];
        kread(ring + ST * R::MAT, kf);
        sc = scores(kf);
      }
      if (n > 0 && n + 2 < tiles) {
        issue(it.t0 + n + 2, std::integral_constant<int, (ST + 2) % 4>{});
        if (n + 3 < tiles) fetch(it.t0 + n + 3);
      }
      if (idle) return;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!B) softmax(sc, tile_bits(it.t0 + n), pf_hold);
      else sc_hold = sc;
      if (n == tiles - 1) {
        if constexpr (B) softmax(sc_hold, tile_bits(it.t0 + n), pf_hold);
        pv_tile(st_c, pf_hold);
      }
    };
    auto run = [&](auto role_c) OOO_INLINE {
      int n = 0;
      for (; n + 4 <= tiles; n += 4) {
        body(role_c, n, I0{});
        body(role_c, n + 1, I1{});
        body(role_c, n + 2, I2{});
        body(role_c, n + 3, I3{});
      }
      if (n < tiles) body(role_c, n, I0{});
      if (n + 1 < tiles) body(role_c, n + 1, I1{});
      if (n + 2 < tiles) body(role_c, n + 2, I2{});
    };
    if (kh0 == 0) run(std::false_type{});
    else run(std::true_type{});
  } else {
    // narrow: half-tiles first, first + 8, ... of this wave
    const int h1 = min(2 * it.t1, (it.limit + 31) / 32);
    uint8_t* const mine = ring + wave * R::MAT;  // K half-tile, then V
    const uint32_t kd = __builtin_amdgcn_readfirstlane(lds_addr(mine)), vd = kd + HB;
    int id0 = 0, id1 = 0;
    auto fetch = [&](int h) OOO_INLINE {
      id0 = pages.at(32 * h, bad);
      id1 = pages.at(min(32 * h + 16, it.limit - 1), bad);
    };
    auto issue = [&](const uint16_t* pool, int h, uint32_t dst) OOO_INLINE {
      const int lo = 32 * h, n = it.limit - lo;
#pragma unroll
      for (int x = 0; x < HI; ++x)
        copy_rows(pool, min(x * R::RPI, n - 1) < 16 ? id0 : id1, lo, n, x * R::RPI, dst + x * 1024);
    };
    int h = 2 * it.t0 + wave;
    if (h < h1) {
      fetch(h);
      issue(kp, h, kd);
      issue(vp, h, vd);
    }
    queries_here();
    for (; h < h1; h += NW) {
      const bool more = h + NW < h1;
      bf16x8 kf[D / 16], vv[2][D / 32], pf[2];
      wait_vmcnt<HI>();  // K is here, V on its way
      kread(mine, kf);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) {
        fetch(h + NW);
        issue(kp, h + NW, kd);
      }
      f32x16 sc = scores(kf);
      const int lo = 32 * h;
      softmax(sc, lo + 32 <= all ? ~0u : (uint32_t)seen(p, it, i, (int)row, lo), pf);
      if (more) wait_vmcnt<HI>();
      else wait_vmcnt<0>();
      vread(mine + HB, 0, vv[0]);
      vread(mine + HB, 1, vv[1]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) issue(vp, h + NW, vd);
      pv(vv[0], pf[0]);
      pv(vv[1], pf[1]);
    }
  }

  // A value of V that is not finite counts only for the rows that give its key
  // a weight, but the products multiply it by the zeros of the others, and
  // zero times it is NaN.  So a wave whose sums are not finite adds its keys
  // once more, one by one, without those of weight zero.
  if (!idle) {
    float z = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 16; ++j) z = __builtin_fmaf(oacc[dt][j], 0.f, z);
    if (__any(!(z == 0.f))) {
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      l_run = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = f32x16{};
      const int step = wide ? 2 : NW;
      for (int h = 2 * it.t0 + (wide ? kh0 : wave); h < 2 * it.t1 && 32 * h < it.limit; h += step) {
        const uint64_t bits = seen(p, it, i, (int)row, 32 * h);
#pragma unroll 1
        for (int j = 0; j < 32 && 32 * h + j < it.limit; ++j) {
          const int t = 32 * h + j;
          const long long base = page_base(pages.at(t, bad), t & in_page);
          float s = 0.f;
#pragma unroll
          for (int dk = 0; dk < D / 16; ++dk) {
            const bf16x8 kk = as_bf16x8(ld16(kp + base + 16 * dk + 8 * u));
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)kk[e], (float)qf[dk][e], s);
          }
          s += shfl_xor_f(s, 32);
          const float w = (bits >> j) & 1 ? __builtin_amdgcn_exp2f(fmaf(s, a.scale_log2e, -m_use)) : 0.f;
          if (w == 0.f) continue;
          if (u == 0) l_run += w;
#pragma unroll
          for (int q = 0; q < NP; ++q) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(vp + base + 8 * q + 4 * u);
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
  if (__any(bad)) bad_s = 1;
  __syncthreads();  // the ring is free, bad_s complete
  auto piece = [&](int q) OOO_INLINE {
    return f32x4{oacc[q / 4][4 * (q % 4)], oacc[q / 4][4 * (q % 4) + 1], oacc[q / 4][4 * (q % 4) + 2],
                 oacc[q / 4][4 * (q % 4) + 3]};
  };
  uint16_t* const orow = (uint16_t*)a.out + (row * p.Hq + hq) * D + 4 * u;
  auto put = [&](int q, f32x4 o, float inv) OOO_INLINE {
    u32x2 pk;
    pk[0] = pack_bf16x2(o[0] * inv, o[1] * inv);
    pk[1] = pack_bf16x2(o[2] * inv, o[3] * inv);
    *reinterpret_cast<u32x2*>(orow + 8 * q) = pk;
  };
  const bool direct = it.flags & kDirect;
  const size_t sl = (size_t)(it.slot + rg) * p.Hkv + g;
  f32x4* const po = reinterpret_cast<f32x4*>(a.part_o) + sl * NP * 64 + lane;
  f32x2_t* const pml = reinterpret_cast<f32x2_t*>(a.part_ml) + sl * 32 + c;
  if (!direct && it.slot + (it.nq + 31) / 32 > a.max_slots) return;
  if (wide) {
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
    if (bad_s) l_tot = __builtin_nanf("");
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
  } else {
    // join the eight waves: wave w adds up pieces w NP / 8 ..
    uint8_t* const mine = ring + wave * R::MAT;
    float* const ml = reinterpret_cast<float*>(mwords);  // [wave][32] (m, l)
#pragma unroll
    for (int q = 0; q < NP; ++q) *reinterpret_cast<f32x4*>(mine + (q * 64 + lane) * 16) = piece(q);
    if (u == 0) *reinterpret_cast<f32x2_t*>(ml + (wave * 32 + c) * 2) = f32x2_t{m_run, l_tot};
    __syncthreads();
    float wm[NW], wl[NW], mn = -INFINITY, den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const f32x2_t x = *reinterpret_cast<const f32x2_t*>(ml + (w * 32 + c) * 2);
      wm[w] = x[0];
      wl[w] = x[1];
      mn = __builtin_fmaxf(mn, x[0]);
    }
    const float base = mn == -INFINITY ? 0.f : mn;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      wm[w] = __builtin_amdgcn_exp2f(wm[w] - base);
      den += wm[w] * wl[w];
    }
    if (bad_s) den = __builtin_nanf("");
    const float inv = den == 0.f ? 0.f : 1.f / den;
#pragma unroll
    for (int x = 0; x < NP / NW; ++x) {
      const int q = wave * (NP / NW) + x;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const f32x4 ow = *reinterpret_cast<const f32x4*>(ring + w * R::MAT + (q * 64 + lane) * 16);
        if (wm[w] > 0.f) o += ow * wm[w];
      }
      if (!on) continue;
      if (direct) put(q, o, inv);
      else po[q * 64] = o;
    }
    if (!direct && on && wave == 0 && u == 0) *pml = f32x2_t{mn, den};
  }
}

}  // namespace ooo
