// Rows of a batch into and inside cache pages.
//
//  * ooo_paged_append   per-head RMSNorm of q and k, rotation at the row's
//                       position, q to [rows][Hq][D], k and v to the pages
//  * ooo_paged_compact  the accepted rows of every sequence moved together
#include "paged.h"
#include "rope.h"
#include "vec16.h"

namespace ooo {
namespace {

// ------------------------------------------------------------------ append
// x <- x / sqrt(mean(x^2) + eps) w per head, then the rotate-half pairs
// (x_j, x_{j + D/2}) turned by (shared + len + depth) theta^(-2j/D).  A lane
// holds 16 bytes of each half of a head, so a wave takes 64 / (D / 2 / N)
// heads of a row (8 of 128 in bf16) and a norm is a sum over 4 to 16
// neighbouring lanes.  The angles are the same for all heads of a row: lane j
// computes pair j's (in double, rope.h) and the lanes fetch theirs through
// LDS.  Waves of one block take the row's head groups.  Bound by HBM: 257 MB of
// 10k rows of 48 heads of 128 in 43 us, 6 TB/s.
constexpr int kAppendWaves = 4;

template <class T, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void append_kernel(
    Paged p, const T* __restrict__ qkv, long long ld, const T* __restrict__ q_norm, const T* __restrict__ k_norm,
    float eps, const int32_t* __restrict__ depth, RopeFreq fr, T* __restrict__ q_out, T* __restrict__ k_pages,
    T* __restrict__ v_pages) {
  using V = Vec16<T>;
  constexpr int N = V::N, HALF = D / 2, LPH = HALF / N, HPW = 64 / LPH;
  __shared__ __attribute__((aligned(16))) float cs_s[kAppendWaves][HALF], sn_s[kAppendWaves][HALF];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x, nh = p.Hq + 2 * p.Hkv;
  const int h0 = ((int)blockIdx.y * kAppendWaves + wave) * HPW;  // first head of this wave
  if (h0 >= nh) return;
  const int h = h0 + lane / LPH, j0 = (lane % LPH) * N;
  const bool on = h < nh;
  const T* src = qkv + (size_t)r * ld + (size_t)min(h, nh - 1) * D + j0;
  const u32x4 xa = ld16(src), xb = ld16(src + HALF);
  const int R = rows_of(p);
  if (r >= R) return;
  const int b = __builtin_amdgcn_readfirstlane(seq_of_row(p.row_start, p.n_seqs, r, lane));
  const Seq q = seq_of(p, b, R);
  const int len = p.seq_len[b], i = r - q.row0;
  if (i < 0 || i >= q.rows) return;  // no sequence's row
  const long long slot = (long long)len + i;
  const int pos = p.shared_len + len + (depth ? depth[r] : i);
  bool ok = len >= 0 && slot < p.own_cap;
  const int page = ok ? p.table[(size_t)b * p.table_ld + (slot >> p.page_shift)] : -1;
  ok = page >= 0 && page < p.n_pages;

  if (lane < HALF) rope_sincos(pos, fr.f[lane], sn_s[wave][lane], cs_s[wave][lane]);
  __builtin_amdgcn_wave_barrier();
  const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
  float a[N], c[N];
  V::unpack(xa, a);
  V::unpack(xb, c);
  const T* nw = is_q ? q_norm : k_norm;
  if (nw && !is_v) {
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
  u32x4 oa = xa, oc = xb;  // values go in unchanged
  if (!is_v) {
    float ra[N], rc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float cs = cs_s[wave][j0 + e], sn = sn_s[wave][j0 + e];
      ra[e] = a[e] * cs - c[e] * sn;
      rc[e] = c[e] * cs + a[e] * sn;
    }
    oa = V::pack(ra);
    oc = V::pack(rc);
  }
  if (!on || (!is_q && !ok)) return;
  T* dst;
  if (is_q) {
    dst = q_out + ((size_t)r * p.Hq + h) * D;
  } else {
    const int g = is_v ? h - p.Hq - p.Hkv : h - p.Hq;
    const int row = (int)(slot & ((1 << p.page_shift) - 1));
    dst = (is_v ? v_pages : k_pages) + (long long)page * p.page_stride + (((size_t)g << p.page_shift) + row) * D;
  }
  st16(dst + j0, oa);
  st16(dst + HALF + j0, oc);
}

// ----------------------------------------------------------------- compact
// One block per (layer, sequence, KV head, K or V).  A chunk of rows is read
// whole before any of it is written; since path[d] >= d rises strictly, the
// rows that a chunk writes lie before the rows that later chunks read.  Bound
// by HBM: 76 MB of 8 sequences in 36 layers in 17 us, 4.4 TB/s read and written.
constexpr int kMovePasses = 4;

template <int LPR>  // 16-byte pieces of a row
__global__ __launch_bounds__(256) void compact_kernel(Paged p, uint8_t* __restrict__ k, uint8_t* __restrict__ v,
                                                      long long layer_bytes, int elt,
                                                      const int32_t* __restrict__ path,
                                                      const int32_t* __restrict__ accept, int path_cap) {
  constexpr int RPP = 256 / LPR;  // rows of a pass
  const int b = blockIdx.y, g = blockIdx.x >> 1;
  uint8_t* const pool = ((blockIdx.x & 1) ? v : k) + (long long)blockIdx.z * layer_bytes;
  const int L = accept[b];
  const int len = p.seq_len[b], rows = seq_of(p, b, rows_of(p)).rows;
  if (L < 0 || L >= path_cap || len < 0) return;
  const int sub = threadIdx.x % LPR, lr = threadIdx.x / LPR;
  const auto place = [&](int i) -> uint8_t* {  // of new row i, or null
    const long long slot = (long long)len + i;
    if (i < 0 || i >= rows || slot >= p.own_cap) return nullptr;
    const int page = p.table[(size_t)b * p.table_ld + (slot >> p.page_shift)];
    if (page < 0 || page >= p.n_pages) return nullptr;
    const long long row = ((long long)g << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
    return pool + (long long)page * p.page_stride * elt + row * (LPR * 16) + sub * 16;
  };
  for (int d0 = 0; d0 <= L; d0 += RPP * kMovePasses) {
    u32x4 x[kMovePasses];
    uint8_t* dst[kMovePasses];
#pragma unroll
    for (int c = 0; c < kMovePasses; ++c) {
      const int d = d0 + c * RPP + lr;
      const int from = d <= L ? path[(size_t)b * path_cap + d] : -1;
      const uint8_t* src = from == d ? nullptr : place(from);
      dst[c] = src ? place(d) : nullptr;
      if (dst[c]) x[c] = ld16(src);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kMovePasses; ++c)
      if (dst[c]) st16(dst[c], x[c]);
    __syncthreads();
  }
}

template <class T, int D>
void launch_append(const Paged& p, const void* qkv, long long ld, const void* q_norm, const void* k_norm, float eps,
                   const int32_t* depth, const RopeFreq& fr, void* q_out, void* k, void* v, hipStream_t st) {
  constexpr int HPW = 64 / (D / 2 / Vec16<T>::N);
  const int nh = p.Hq + 2 * p.Hkv, groups = (nh + HPW - 1) / HPW;
  const dim3 grid(p.n_rows, (groups + kAppendWaves - 1) / kAppendWaves);
  append_kernel<T, D><<<grid, 64 * kAppendWaves, 0, st>>>(p, (const T*)qkv, ld, (const T*)q_norm, (const T*)k_norm,
                                                          eps, depth, fr, (T*)q_out, (T*)k, (T*)v);
}

}  // namespace
}  // namespace ooo

using namespace ooo;

extern "C" int ooo_paged_append(const ooo_paged_batch* batch, const void* qkv, int64_t qkv_ld, const void* q_norm,
                                const void* k_norm, float eps, const int32_t* depth, double rope_theta, void* q_out,
                                void* k_pages, void* v_pages, void* stream) {
  Paged p{};
  const int rc = check_paged("ooo_paged_append", batch, p);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(qkv && q_out && k_pages && v_pages, OOO_ERR_INVALID, "ooo_paged_append: null pointer");
  OOO_REQUIRE(rope_theta > 0.0 && eps >= 0.f, OOO_ERR_INVALID, "ooo_paged_append: rope_theta must be > 0, eps >= 0");
  const int D = batch->head_dim, per16 = batch->dt == OOO_BF16 ? 8 : 4;
  OOO_REQUIRE(qkv_ld >= (int64_t)(p.Hq + 2 * p.Hkv) * D, OOO_ERR_INVALID,
              "ooo_paged_append: qkv_ld %lld below the row's %lld elements", (long long)qkv_ld,
              (long long)(p.Hq + 2 * p.Hkv) * D);
  OOO_REQUIRE(qkv_ld % per16 == 0 && aligned16(qkv) && aligned16(q_out) && aligned16(k_pages) && aligned16(v_pages) &&
                  aligned16(q_norm) && aligned16(k_norm),
              OOO_ERR_UNSUPPORTED, "ooo_paged_append: a pointer or qkv_ld is not a multiple of 16 bytes");
  const RopeFreq fr = rope_freq(rope_theta, D);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (batch->dt == OOO_BF16 && D == 128)
    launch_append<uint16_t, 128>(p, qkv, qkv_ld, q_norm, k_norm, eps, depth, fr, q_out, k_pages, v_pages, st);
  else if (batch->dt == OOO_BF16)
    launch_append<uint16_t, 64>(p, qkv, qkv_ld, q_norm, k_norm, eps, depth, fr, q_out, k_pages, v_pages, st);
  else if (D == 128)
    launch_append<float, 128>(p, qkv, qkv_ld, q_norm, k_norm, eps, depth, fr, q_out, k_pages, v_pages, st);
  else
    launch_append<float, 64>(p, qkv, qkv_ld, q_norm, k_norm, eps, depth, fr, q_out, k_pages, v_pages, st);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "ooo_paged_append: launch failed: %s", hipGetErrorString(e));
  return ooo::ok();
}

extern "C" int ooo_paged_compact(const ooo_paged_batch* batch, void* k_pages, void* v_pages, int32_t n_layers,
                                 int64_t layer_stride, const int32_t* path, const int32_t* accept_len,
                                 int32_t path_cap, void* stream) {
  Paged p{};
  const int rc = check_paged("ooo_paged_compact", batch, p);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(k_pages && v_pages && path && accept_len, OOO_ERR_INVALID, "ooo_paged_compact: null pointer");
  OOO_REQUIRE(n_layers >= 1 && path_cap >= 1, OOO_ERR_INVALID, "ooo_paged_compact: n_layers and path_cap must be >= 1");
  OOO_REQUIRE(n_layers == 1 || layer_stride >= 1, OOO_ERR_INVALID, "ooo_paged_compact: layer_stride must be >= 1");
  OOO_REQUIRE(n_layers <= 65535, OOO_ERR_UNSUPPORTED, "ooo_paged_compact: n_layers %d above 65535", n_layers);
  const int elt = batch->dt == OOO_BF16 ? 2 : 4;
  OOO_REQUIRE(layer_stride * elt % 16 == 0 && aligned16(k_pages) && aligned16(v_pages), OOO_ERR_UNSUPPORTED,
              "ooo_paged_compact: a pointer or layer_stride is not a multiple of 16 bytes");
  const dim3 grid(2 * p.Hkv, p.n_seqs, n_layers);
  const long long lb = layer_stride * elt;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  uint8_t *k = (uint8_t*)k_pages, *v = (uint8_t*)v_pages;
  switch (batch->head_dim * elt / 16) {
    case 8: compact_kernel<8><<<grid, 256, 0, st>>>(p, k, v, lb, elt, path, accept_len, path_cap); break;
    case 16: compact_kernel<16><<<grid, 256, 0, st>>>(p, k, v, lb, elt, path, accept_len, path_cap); break;
    default: compact_kernel<32><<<grid, 256, 0, st>>>(p, k, v, lb, elt, path, accept_len, path_cap); break;
  }
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "ooo_paged_compact: launch failed: %s", hipGetErrorString(e));
  return ooo::ok();
}
