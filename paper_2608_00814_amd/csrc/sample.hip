// One token from each row of logits.
//
// With a row's tokens ordered by (logit descending, index ascending) and
// weights w = exp((x - max) / T), every question the draw asks is the same
// one: at which place of that order does a running count or a running sum of
// weights reach a value?
//   top-k    the sum S_k at count k
//   top-p    the count n_p at which the sum reaches top_p S_k
//   min-p    n_m, the number of weights of at least min_p
//   kept     the sum W at count n = min(k, n_p, n_m)
//   draw     the token at which the sum exceeds u W
// So no row is sorted.  A histogram over (max - x) / T (count and weight of
// each bin) finds the bins in which the places lie, the tokens of those bins
// alone are gathered and sorted, and running sums over them, on top of the
// bins' before, answer the questions in turn.
//
// Weights are whole numbers, round(w 2^s) with s = 62 - ceil(log2 vocab):
// sums are exact, so the order of additions (the atomics') does not change
// results, and a weight is as exact as 2^-42 of the largest at least (float32
// weights would move the borders by their rounding: of 152064 equal-ish
// tokens one row in 50 would draw a neighbour).
#include <algorithm>

#include "device_common.h"
#include "ooo_batch.h"
#include "ooo_internal.h"

namespace ooo {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 1024;        // the last one holds what lies past the range
constexpr float kRange = 32.f;     // (max - x) / T of the bins: weights above exp(-32) < 2^-46
constexpr int kGather = 4096;      // tokens of the bins that are looked at closely
constexpr int kThreads = 1024;

struct SampleArgs {
  const void* logits;
  long long ld;
  int vocab, shift;  // weights are scaled by 2^shift
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* ids;
  float* prob;
  int32_t* kept;
};

__device__ __forceinline__ float logit(const float* p) { return *p; }
__device__ __forceinline__ float logit(const uint16_t* p) { return bf16_bits_to_f32(*p); }

// A token's logit with NaN as -inf and -0 as 0.
__device__ __forceinline__ float clean(float x) { return x == x ? x + 0.f : -INFINITY; }

// Order of logits as whole numbers, the largest logit first.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? b : ~b & 0x7FFFFFFFu;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k : ~k & 0x7FFFFFFFu);
}

// A row's settings.
struct Row {
  float M, inv_t;       // largest logit, 1 / T for the bins
  double T, floor_z;    // T and log(min_p) (-inf: no floor)
  int k, shift;
  double top_p, u;
  __device__ __forceinline__ double z(float x) const {
    const double y = x == M ? 0.0 : ((double)x - (double)M) / T;
    return y == y ? y : -INFINITY;  // below an infinite maximum at an infinite T
  }
  __device__ __forceinline__ int bin(float x) const {
    const float y = x == M ? 0.f : (M - x) * inv_t;
    return y < kRange ? (int)(y * ((kBins - 1) / kRange)) : kBins - 1;
  }
  __device__ __forceinline__ u64 weight(float x) const {
    const double y = z(x);
    return y < -44.0 ? 0ull : (u64)rint(ldexp(exp(y), shift));
  }
};

__device__ __forceinline__ Row row_of(const SampleArgs& a, int r, float M) {
  Row s;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  const bool greedy = !(t > 0.f);
  s.M = M;
  s.T = greedy ? 1.0 : (double)t;
  s.inv_t = greedy ? 1.f : 1.f / t;
  const int k = a.top_k ? a.top_k[r] : 0;
  s.k = greedy ? 1 : k > 0 ? k : a.vocab;
  const float tp = a.top_p ? a.top_p[r] : 1.f;
  s.top_p = tp < 1.f ? fmax((double)tp, 0.0) : tp >= 1.f ? 1.0 : 0.0;
  const float mp = a.min_p ? a.min_p[r] : 0.f;
  s.floor_z = mp > 0.f ? log((double)mp) : -INFINITY;
  const float u = a.u[r];
  s.u = u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0;
  s.shift = a.shift;
  return s;
}

// ---- workgroup helpers (every thread calls them)
__device__ __forceinline__ float block_max(float v, float* sh) {
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, shfl_xor_f(v, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
  for (int w = 1; w < kThreads / 64; ++w) v = fmaxf(v, sh[w]);
  return v;
}
// inclusive scan over the threads; `total` goes to all
__device__ __forceinline__ u64 block_scan(u64 v, u64& total, u64* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int off = 1; off < 64; off <<= 1) {
    const u64 o = __shfl_up(v, off, 64);
    if (lane >= off) v += o;
  }
  __syncthreads();
  if (lane == 63) sh[wave] = v;
  __syncthreads();
  u64 before = 0;
  total = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w == wave) before = total;
    total += sh[w];
  }
  return v + before;
}

struct Found {
  u64 count, weight;  // of the tokens before the value
  uint32_t key;       // the value
  u64 ties;           // tokens of that value
};

// The place of the row at which the running count exceeds `target`
// (by_weight false) or the running weight does (true; > or >= by `reach`),
// found digit by digit over the keys: four passes over the row.  For rows
// whose close bins hold more than fits (many equal logits).
template <class T>
__device__ Found radix_find(const T* x, int V, const Row& s, bool by_weight, u64 target, u64* hw, u64* hc, u64* sh) {
  Found f{0, 0, 0, 0};
  for (int level = 0; level < 4; ++level) {
    const int sft = 24 - 8 * level;
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += kThreads) hw[i] = hc[i] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < V; i0 += kThreads) {
      const int i = i0 + threadIdx.x;
      const float v = i < V ? clean(logit(x + i)) : -INFINITY;
      const uint32_t k = key_of(v);
      const bool in = v > -INFINITY && (level == 0 || (k >> (sft + 8)) == (f.key >> (sft + 8)));
      const int d = in ? (int)((k >> sft) & 255) : -1;
      u64 w = in ? s.weight(v) : 0;
      const u64 lanes = __ballot(in);
      if (!lanes) continue;
      // one digit in the whole wave (the usual case at the first levels):
      // one addition for it
      const int d0 = __builtin_amdgcn_readlane(d, __builtin_ctzll(lanes));
      if (__all(!in || d == d0)) {
        for (int off = 32; off > 0; off >>= 1) w += __shfl_xor(w, off, 64);
        if ((threadIdx.x & 63) == 0) {
          atomicAdd(&hw[d0], w);
          atomicAdd(&hc[d0], (u64)__popcll(lanes));
        }
      } else if (in) {
        atomicAdd(&hw[d], w);
        atomicAdd(&hc[d], 1ull);
      }
    }
    __syncthreads();
    u64 c = threadIdx.x < 256 ? hc[threadIdx.x] : 0, w = threadIdx.x < 256 ? hw[threadIdx.x] : 0;
    u64 tc, tw;
    const u64 ic = block_scan(c, tc, sh), iw = block_scan(w, tw, sh);
    const u64 at = by_weight ? f.weight + iw : f.count + ic, was = by_weight ? at - w : at - c;
    __shared__ Found got;
    if (threadIdx.x < 256 && c > 0 && at > target && was <= target)
      got = Found{f.count + ic - c, f.weight + iw - w, f.key | (uint32_t)threadIdx.x << sft, c};
    __syncthreads();
    f = got;
  }
  return f;
}

// One workgroup per row.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ u64 bin_w[kBins];
  __shared__ uint32_t bin_c[kBins];
  __shared__ u64 cand[kGather];  // (key, index), sorted
  __shared__ u64 sh[32];
  __shared__ float shf[kThreads / 64];
  __shared__ u64 res[4];
  __shared__ uint32_t n_cand, n_floor;
  const int r = blockIdx.x, tid = threadIdx.x, V = a.vocab;
  const T* x = (const T*)a.logits + (long long)r * a.ld;

  float M = -INFINITY;
  for (int i = tid; i < V; i += kThreads) M = fmaxf(M, clean(logit(x + i)));
  M = block_max(M, shf);
  if (M == -INFINITY) {
    if (tid == 0) {
      a.ids[r] = -1;
      if (a.prob) a.prob[r] = 0.f;
      if (a.kept) a.kept[r] = 0;
    }
    return;
  }
  const Row s = row_of(a, r, M);

  // histogram
  for (int i = tid; i < kBins; i += kThreads) bin_w[i] = 0, bin_c[i] = 0;
  if (tid == 0) n_cand = n_floor = 0;
  __syncthreads();
  uint32_t over_floor = 0;
  for (int i = tid; i < V; i += kThreads) {
    const float v = clean(logit(x + i));
    if (v == -INFINITY) continue;
    const int b = s.bin(v);
    atomicAdd(&bin_c[b], 1u);
    over_floor += s.z(v) >= s.floor_z;
    if (b < kBins - 1) atomicAdd(&bin_w[b], s.weight(v));
  }
  atomicAdd(&n_floor, over_floor);
  __syncthreads();
  // counts and weights before each bin (thread b: bin b)
  u64 live, total;
  const u64 c_in = bin_c[tid], w_in = bin_w[tid];
  const u64 c_to = block_scan(c_in, live, sh), w_to = block_scan(w_in, total, sh);
  const u64 c_at = c_to - c_in, w_at = w_to - w_in;
  const u64 k = min((u64)s.k, live), floor_n = max((u64)n_floor, 1ull);
  // Bins that the places can lie in.  Where a bin holds a place, the sum there
  // is known to within the bin's weight; the places that depend on it lie
  // between the bins of the two ends.  Nothing in the last bin weighs anything.
  __shared__ int need[kBins];
  __shared__ u64 lohi[2];
  const auto bounds = [&](u64 count) {  // weight at `count`: from, to
    __syncthreads();
    if (c_at < count && count <= c_to) {
      lohi[0] = count == c_to ? w_to : w_at;
      lohi[1] = w_to;
      if (count < c_to && tid < kBins - 1) need[tid] = 1;
    }
    __syncthreads();
  };
  need[tid] = 0;
  bounds(k);
  u64 n_lo = k, n_hi = k;  // bounds of the kept count
  if (s.top_p < 1.0) {
    const double lo = s.top_p * (double)lohi[0], hi = s.top_p * (double)lohi[1];
    __syncthreads();
    if (tid == 0) res[0] = 1, res[1] = hi > 0.0 ? k : 1;
    __syncthreads();
    if (c_in && (double)w_to >= lo && (double)w_at <= hi) need[tid] = 1;
    if (c_in && (double)w_to >= lo && (double)w_at < lo) res[0] = c_at + 1;
    if (c_in && (double)w_to >= hi && (double)w_at < hi) res[1] = c_to;
    __syncthreads();
    n_lo = min(k, res[0]);
    n_hi = min(k, res[1]);
  }
  n_lo = max(min(n_lo, floor_n), 1ull);
  n_hi = max(min(n_hi, floor_n), 1ull);
  bounds(n_lo);
  const double d_lo = s.u * (double)lohi[0];
  bounds(n_hi);
  const double d_hi = s.u * (double)lohi[1];
  if (c_in && (double)w_to > d_lo && (double)w_at <= d_hi) need[tid] = 1;
  __syncthreads();
  // place of each needed bin among the gathered tokens
  u64 gathered;
  const u64 g_to = block_scan(need[tid] ? c_in : 0, gathered, sh);
  __shared__ uint32_t first_of[kBins];
  first_of[tid] = (uint32_t)(g_to - (need[tid] ? c_in : 0));
  __shared__ u64 w_before[kBins];
  __shared__ uint32_t c_before[kBins];
  w_before[tid] = w_at;
  c_before[tid] = (uint32_t)c_at;
  __syncthreads();

  float best;     // the drawn token's logit
  int id = -1;
  u64 n, W;
  if (gathered <= kGather) {
    for (int i = tid; i < V; i += kThreads) {
      const float v = clean(logit(x + i));
      if (v == -INFINITY || !need[s.bin(v)]) continue;
      cand[atomicAdd(&n_cand, 1u)] = (u64)key_of(v) << 32 | (uint32_t)i;
    }
    int size = 2;
    while (size < (int)gathered) size *= 2;
    __syncthreads();
    for (int i = (int)gathered + tid; i < size; i += kThreads) cand[i] = ~0ull;
    for (int len = 2; len <= size; len *= 2)
      for (int j = len / 2; j > 0; j /= 2) {
        __syncthreads();
        for (int i = tid; i < size / 2; i += kThreads) {
          const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
          const u64 p = cand[lo], q = cand[hi];
          if ((p > q) == ((lo & len) == 0)) cand[lo] = q, cand[hi] = p;
        }
      }
    __syncthreads();
    // running count and weight at each gathered token: 4 a thread in a row
    constexpr int PT = kGather / kThreads;
    u64 w[PT], mine = 0;
    int bin[PT];
#pragma unroll
    for (int e = 0; e < PT; ++e) {
      const int i = tid * PT + e;
      const float v = i < (int)gathered ? of_key((uint32_t)(cand[i] >> 32)) : 0.f;
      bin[e] = i < (int)gathered ? s.bin(v) : -1;
      w[e] = i < (int)gathered && bin[e] < kBins - 1 ? s.weight(v) : 0;
      mine += w[e];
    }
    u64 all;
    u64 at = block_scan(mine, all, sh) - mine;
    // the running sum where each bin begins, to be taken off
    __shared__ u64 start[kBins];
    u64 run[PT];
#pragma unroll
    for (int e = 0; e < PT; ++e) {
      if (bin[e] >= 0 && (uint32_t)(tid * PT + e) == first_of[bin[e]]) start[bin[e]] = at;
      at += w[e];
      run[e] = at;
    }
    __syncthreads();
    u64 cnt[PT];
#pragma unroll
    for (int e = 0; e < PT; ++e)
      if (bin[e] >= 0) {
        run[e] += w_before[bin[e]] - start[bin[e]];
        cnt[e] = c_before[bin[e]] + (tid * PT + e - first_of[bin[e]]) + 1;
      }
    const auto sum_at = [&](u64 count) -> u64 {
      __syncthreads();
      if (c_at < count && count <= c_to) res[2] = w_to;  // a bin's end, or nothing more weighs anything
      __syncthreads();
#pragma unroll
      for (int e = 0; e < PT; ++e)
        if (bin[e] >= 0 && cnt[e] == count) res[2] = run[e];
      __syncthreads();
      return res[2];
    };
    n = k;
    if (s.top_p < 1.0) {
      const double target = s.top_p * (double)sum_at(k);
      if (tid == 0) res[3] = target > 0.0 ? k : 1;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < PT; ++e)
        if (bin[e] >= 0 && (double)run[e] >= target && (double)(run[e] - w[e]) < target) res[3] = cnt[e];
      __syncthreads();
      n = min(n, res[3]);
    }
    n = max(min(n, floor_n), 1ull);
    W = sum_at(n);
    const double target = s.u * (double)W;
    if (tid == 0) res[3] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PT; ++e)
      if (bin[e] >= 0 && (double)run[e] > target && (double)(run[e] - w[e]) <= target) res[3] = tid * PT + e;
    __syncthreads();
    const u64 c = cand[res[3]];
    id = (int)(uint32_t)c;
    best = of_key((uint32_t)(c >> 32));
  } else {
    // too many tokens in the close bins: by digits over the whole row
    const auto sum_at = [&](u64 count) -> u64 {
      if (count >= live) return total;
      const Found f = radix_find(x, V, s, false, count - 1, bin_w, cand, sh);
      return f.weight + (count - f.count) * s.weight(of_key(f.key));
    };
    n = k;
    if (s.top_p < 1.0) {
      const double target = s.top_p * (double)sum_at(k);
      u64 np = 1;
      if (target > 0.0) {
        // the first running weight >= target is the first > ceil(target) - 1
        const u64 t = (u64)ceil(target);
        const Found f = radix_find(x, V, s, true, t - 1, bin_w, cand, sh);
        const u64 w = s.weight(of_key(f.key));
        np = f.count + (t - f.weight + w - 1) / w;
      }
      n = min(n, np);
    }
    n = max(min(n, floor_n), 1ull);
    W = sum_at(n);
    const u64 t = (u64)floor(s.u * (double)W);
    const Found f = radix_find(x, V, s, true, t, bin_w, cand, sh);
    best = of_key(f.key);
    const u64 want = (t - f.weight) / s.weight(best);  // this many equal ones come before it
    u64 seen = 0;
    for (int i0 = 0; i0 < V; i0 += kThreads) {
      const int i = i0 + tid;
      const bool eq = i < V && clean(logit(x + i)) == best;
      u64 here;
      const u64 to = block_scan(eq, here, sh);
      if (eq && seen + to - 1 == want) res[3] = i;
      seen += here;
      if (seen > want) break;
    }
    __syncthreads();
    id = (int)res[3];
  }
  if (tid == 0) {
    a.ids[r] = id;
    if (a.prob) a.prob[r] = (float)(exp(s.z(best)) / ldexp((double)W, -s.shift));
    if (a.kept) a.kept[r] = (int32_t)n;
  }
}

}  // namespace
}  // namespace ooo

using namespace ooo;

extern "C" size_t ooo_sample_workspace(int32_t n_rows, int32_t vocab) {
  if (n_rows < 1 || vocab < 1 || vocab > (1 << 20)) return 0;
  return 16;
}

extern "C" int ooo_sample(const void* logits, int64_t ld, ooo_dtype dt, int32_t n_rows, int32_t vocab,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                          const float* u, int32_t* ids, float* prob, int32_t* kept, void* workspace,
                          size_t ws_bytes, void* stream) {
  OOO_REQUIRE(logits && u && ids && workspace, OOO_ERR_INVALID, "ooo_sample: null pointer");
  OOO_REQUIRE(n_rows >= 1 && vocab >= 1, OOO_ERR_INVALID, "ooo_sample: sizes must be positive");
  OOO_REQUIRE(ld >= vocab, OOO_ERR_INVALID, "ooo_sample: ld %lld below vocab %d", (long long)ld, vocab);
  OOO_REQUIRE(dt == OOO_F32 || dt == OOO_BF16, OOO_ERR_INVALID, "ooo_sample: unknown dtype %d", (int)dt);
  OOO_REQUIRE(vocab <= (1 << 20), OOO_ERR_UNSUPPORTED, "ooo_sample: vocab %d above 2^20", vocab);
  OOO_REQUIRE(ws_bytes >= ooo_sample_workspace(n_rows, vocab), OOO_ERR_CAPACITY,
              "ooo_sample: workspace of %zu bytes needed (got %zu)", ooo_sample_workspace(n_rows, vocab), ws_bytes);
  int log2v = 0;
  while ((1 << log2v) < vocab) ++log2v;
  SampleArgs a{logits, ld, vocab, 62 - log2v, temperature, top_k, top_p, min_p, u, ids, prob, kept};
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dt == OOO_BF16) sample_kernel<uint16_t><<<n_rows, kThreads, 0, st>>>(a);
  else sample_kernel<float><<<n_rows, kThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "ooo_sample: launch failed: %s", hipGetErrorString(e));
  return ooo::ok();
}
