// Pieces of the bf16 attention kernels (tree_attn.hip, paged_attn.hip): the
// LDS DMA, the layout of K and V tiles in LDS and the waits for them.
#pragma once

#include "device_common.h"

namespace ooo {

constexpr int kTile = 64;  // keys of a tile

// swap bits 2 and 3: the K row a lane loads so that S^T lands with eight
// consecutive keys per lane and k-step
__device__ __forceinline__ int sigma(int c) { return (c & ~0xC) | ((c & 4) << 1) | ((c & 8) >> 1); }

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
// Kernel-local lambdas must be inlined: an outlined call would take its
// captures through memory and lose their wave-uniformity (the DMA needs
// scalar operands).
#define OOO_INLINE __attribute__((always_inline))

// LDS DMA of 16 bytes per lane from base + voff (base wave-uniform, voff
// per lane); lane l's bytes land at LDS byte address lds + 16*l (lds
// wave-uniform).  Issued through inline asm so the compiler does not track
// it: it would otherwise make LDS reads of other ring stages wait for every
// DMA in flight.  Kernels wait for their DMA explicitly (vmcnt, then a
// barrier).  M0 holds the LDS base; nothing else in these kernels uses M0.
__device__ __forceinline__ void dma16(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

// Same with the non-temporal (streaming) cache policy, for the K/V tiles:
// each head's K/V stream is read once per row block, and keeping it from
// displacing the rest of the L2 (the queries every split re-reads, the
// partials) measured 16.6 -> 15.5 us per call at the Qwen3-8B shape.
__device__ __forceinline__ void dma16_nt(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

// The same at OFF bytes behind both the source and the LDS address.
template <int OFF>
__device__ __forceinline__ void dma16_nt_at(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3 nt" ::"s"(lds), "v"(voff),
               "s"(base), "n"(OFF)
               : "memory", "m0");
}

// Same for 4 bytes per lane (lane l's dword lands at lds + 4*l).
__device__ __forceinline__ void dma4(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// max of three floats without the NaN canonicalisation fmaxf implies
// (scores are finite or -inf)
__device__ __forceinline__ float max3f(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// s plus the two bf16 values packed in x: their dot product with ones.
__device__ __forceinline__ float add_bf16x2(uint32_t x, float s) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x), __builtin_bit_cast(bf16x2_t, 0x3F803F80u), s,
                                         false);
}

// The end of the wait for a matrix product's result: the compiler knows how
// long a vector instruction of its own has to stay behind the product that it
// reads, but not one in inline asm (max3f), which would read what was there
// before.
__device__ __forceinline__ void settle(f32x16& s) {
  const int t = __builtin_amdgcn_readfirstlane(__float_as_int(s[15]));
  asm volatile("" : "+v"(s) : "s"(t));
}

// LDS ring geometry for one head_dim.  A tile is 64 rows of K and 64 rows of
// V, each row D bf16 values = D/8 16-byte chunks, stored row-major with the
// chunks of a row permuted (swz below).  One 1 KiB DMA instruction copies
// whole contiguous rows (coalesced in global memory).  Every stage of every
// matrix is its own __shared__ array, so the compiler can tell that a DMA
// into one stage does not alias reads of another and adds no waits of its
// own; the kernel waits explicitly (vmcnt, then a barrier).
template <int D>
struct KvRing {
  static constexpr int CH = D / 8;            // chunks per row
  static constexpr int ROWB = 2 * D;          // bytes per row
  static constexpr int MAT = kTile * ROWB;    // bytes of one K or V tile
  static constexpr int NS = 4;                // stages
  static constexpr int DMA_MAT = MAT / 1024;  // DMA instructions per matrix
  static constexpr int RPI = 1024 / ROWB;     // rows per DMA instruction
  static constexpr int GPL = D / 8;           // float4 groups of O^T per lane
  // Physical chunk of logical chunk c in row r.  For D = 128 the two 2-bit
  // halves of r % 16 are swapped and XORed in: the K fragment reads (16
  // lanes, 16 different rows, one chunk) and the V transpose reads (32
  // lanes, 4 consecutive rows x 4 consecutive chunks) both hit distinct banks.
  static __device__ __forceinline__ int swz(int r, int c) {
    if (D == 128) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
    return c ^ (r % CH);
  }
};

// wait until at most `ahead` tiles of `per` DMA instructions are pending
template <int PER, int MAXA>
__device__ __forceinline__ void wait_tiles(int ahead) {
  if (MAXA >= 2 && ahead >= 2) wait_vmcnt<(MAXA >= 2 ? 2 * PER : 0)>();
  else if (ahead == 1) wait_vmcnt<PER>();
  else wait_vmcnt<0>();
}

}  // namespace ooo
