// What the kernels over 8-bit cache pages share: the descriptor as kernels take
// it, its checks, and scales and numbers of a block.
#pragma once

#include "ooo_cache8.h"
#include "paged.h"

namespace ooo {

constexpr int kBlockRows = 32;                // rows of a scale
constexpr int kLeastExp = -100, kMostExp = 119;
constexpr float kMostCode = 448.f;

// One layer of ooo_cache8 by value.
struct Cache8 {
  uint8_t* pages[2];   // K, V
  uint8_t* scales[2];
  long long scale_stride;
  int page_blocks;     // blocks of a page and head
};

// Checks shared by the entry points; fills `p` and the first layer's `c`.
inline int check_cache8(const char* who, const ooo_paged_batch* b, const ooo_cache8* cache, Paged& p, Cache8& c) {
  const int rc = check_paged(who, b, p);
  if (rc != OOO_OK) return rc;
  OOO_REQUIRE(b->page_rows >= kBlockRows, OOO_ERR_UNSUPPORTED, "%s: page_rows %d not supported (32 or more)", who,
              b->page_rows);
  OOO_REQUIRE(b->page_stride % 16 == 0, OOO_ERR_UNSUPPORTED, "%s: page_stride is not a multiple of 16 bytes", who);
  c.page_blocks = b->page_rows / kBlockRows;
  if (!cache) return OOO_OK;  // the size queries and the plan
  OOO_REQUIRE(cache->k_pages && cache->v_pages && cache->k_scales && cache->v_scales, OOO_ERR_INVALID,
              "%s: a pool of the cache is null", who);
  OOO_REQUIRE(cache->n_layers >= 1, OOO_ERR_INVALID, "%s: n_layers must be >= 1", who);
  OOO_REQUIRE(cache->n_layers <= 65535, OOO_ERR_UNSUPPORTED, "%s: n_layers %d above 65535", who, cache->n_layers);
  const int64_t least = (int64_t)b->n_kv_heads * c.page_blocks;
  OOO_REQUIRE(cache->scale_stride >= least, OOO_ERR_INVALID, "%s: scale_stride %lld below a page's %lld scales", who,
              (long long)cache->scale_stride, (long long)least);
  OOO_REQUIRE(cache->n_layers == 1 || (cache->layer_stride >= 1 && cache->scale_layer_stride >= 1), OOO_ERR_INVALID,
              "%s: layer strides must be >= 1", who);
  OOO_REQUIRE((cache->n_layers == 1 || cache->layer_stride % 16 == 0) && aligned16(cache->k_pages) &&
                  aligned16(cache->v_pages),
              OOO_ERR_UNSUPPORTED, "%s: a pool or layer_stride is not a multiple of 16 bytes", who);
  c.pages[0] = (uint8_t*)cache->k_pages;
  c.pages[1] = (uint8_t*)cache->v_pages;
  c.scales[0] = (uint8_t*)cache->k_scales;
  c.scales[1] = (uint8_t*)cache->v_scales;
  c.scale_stride = cache->scale_stride;
  return OOO_OK;
}

inline int take_layer(const char* who, const ooo_cache8* cache, int32_t layer, Cache8& c) {
  OOO_REQUIRE(layer >= 0 && layer < cache->n_layers, OOO_ERR_INVALID, "%s: layer %d of %d", who, layer,
              cache->n_layers);
  for (int x = 0; x < 2 && layer > 0; ++x) {
    c.pages[x] += layer * cache->layer_stride;
    c.scales[x] += layer * cache->scale_layer_stride;
  }
  return OOO_OK;
}

// The least e from kLeastExp to kMostExp with x <= 448 * 2^e, for finite x >= 0:
// 448 is 1.75 * 2^8, so of x = m 2^k, 1 <= m < 2, e is k - 8, or k - 7 where m
// is above 1.75 (subnormal x are below all bounds).
__device__ __forceinline__ int exp_for(float x) {
  const uint32_t b = __float_as_uint(x);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kLeastExp), kMostExp);
}
// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// A block's scale as float32 (2^-127 as 0).
__device__ __forceinline__ float scale_of(const uint8_t* p) { return __uint_as_float((uint32_t)*p << 23); }

// |x|, or 0 where x is not finite: it asks for no scale.
__device__ __forceinline__ float size_of(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

// Two or four values times 2^-e (`down`) as e4m3, rounded to nearest even.  What
// is finite is bounded first (the conversion makes NaN of what does not fit, as
// of infinities and NaN).
__device__ __forceinline__ float bounded(float x) {
  return fabsf(x) < INFINITY ? __builtin_fminf(__builtin_fmaxf(x, -kMostCode), kMostCode) : __builtin_nanf("");
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float down) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(bounded(a * down), bounded(b * down), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bounded(c * down), bounded(d * down), w, true);
}
// Four numbers times `up`, a power of two.
__device__ __forceinline__ void values4(uint32_t w, float up, float (&f)[4]) {
  const f32x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, up, false);
  const f32x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, up, true);
  f[0] = lo[0], f[1] = lo[1], f[2] = hi[0], f[3] = hi[1];
}
// Four numbers under a scale that is 2^k times theirs, k >= 0.  Past 24 halvings
// the largest is below half of the least one.
__device__ __forceinline__ uint32_t fewer4(uint32_t w, int k) {
  float f[4];
  values4(w, pow2(-min(k, 24)), f);
  return codes4(f[0], f[1], f[2], f[3], 1.f);
}

}  // namespace ooo
