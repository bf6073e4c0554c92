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
// So no row is sorted.  A histogram over log2 w (count and weight of each bin)
// finds the few bins in which the places lie, the tokens of those bins alone
// are gathered and sorted, and running sums over them, on top of the bins'
// before, answer the questions in turn.
//
// Weights are whole numbers, round(w 2^shift): sums are exact, so the order of
// additions (the atomics') does not change results.  The exponential is
// computed in double: with float32's rounding, of 152064 nearly equal tokens
// one draw in 50 would go to a neighbour.
//
// Rows of up to kOneBlock tokens are one workgroup's work: one launch, where
// chunks take four (240 rows of 11053: 24 us, 46 in chunks; 17 rows of 17940:
// 27 and 34).  Near the bound it depends on the settings and the rows: of 32000
// tokens, 1, 28 and 100 rows with top-k 50 take 11, 12 and 13 us, and 16, 18 and
// 25 in chunks; with top-p alone 33, 35 and 35, and 25, 30 and 48.  Longer ones
// are cut into chunks over many workgroups.  The first launch finds the largest
// logit and those of up to kGroups disjoint groups of tokens.
//  * With top-k (or greedily), no token below the k-th largest of the groups'
//    largest logits can be kept, and only the groups that reach that are read
//    again: the row's workgroup of the last launch gathers their tokens, a few
//    more than k, sorts them and answers from them alone.
//  * Other rows need the two launches between: the histogram and the
//    gathering; they come from HBM once and from the last-level cache twice.
// Where the bins that are needed hold more than kGather tokens, one workgroup
// finds the places digit by digit over the whole row, up to eighteen passes.
// Many equal logits do that, and so do flat ones: a bin is 0.0156 T wide, and of
// 151936 normal logits with standard deviation 1, T 1 and top-p 0.9 without
// top-k more lie in them.  That row takes 1.3 ms (25 to 50 us with a standard
// deviation of 2.5 to 1.28), 64 such rows 1.5 and 256 rows 2.1.
// (Left to the last workgroup of a row to finish, the answers cost more than
// their launch: each workgroup's release and acquire across the XCDs' caches
// took 256 rows of 152064 from 183 to 255 us.)
//
// 256 rows of 152064 float32 logits take 120 us: the largest logits 26 (HBM, 6
// TB/s), the histogram 37 (the exponential and LDS atomics) and the gathering 32
// (the search for the bins in every workgroup) of the third of the rows that
// have no top-k, the answers 23, one workgroup a row.  Rows of 1024 tokens
// take 12 us and the answer of a long one with top-k 14: some fifteen barriers,
// and instructions that run once each and are waited for (the search for the
// bins 8400 cycles, the ordering of 200 tokens 6100, the histogram 2600).
#include "device_common.h"
#include "ooo_batch.h"
#include "ooo_internal.h"

namespace ooo {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 2048;
constexpr int kLast = kBins - 1;     // the bin of what lies past the range and weighs nothing
constexpr double kRange = 46.0;      // log2 of the least weight of the other bins
constexpr int kGather = 2048;        // tokens of the bins that are looked at closely
constexpr int kReplicas = 2;         // of a chunk's histogram, by lane: fewer lanes meet in one bin
constexpr int kOneBlock = 32768;      // tokens
constexpr int kGroups = 4096;        // groups of a long row, at most
constexpr int kFlat = 1024;          // tokens that are answered from without bins
constexpr int kFlatK = 512;          // the largest top-k that goes by its groups
constexpr int kThreads = 512;

// A row's scratch.
struct RowWork {
  u64 w[kBins];
  uint32_t c[kBins];
  uint32_t gathered, over_floor;
  float group_max[kGroups];
  u64 cand[kGather];
};

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
  RowWork* work;
  int chunk, chunks;  // tokens of a chunk, chunks of a row
  int lanes;          // threads of a chunk whose tokens make a group
};

// A token's logit with NaN as -inf and -0 as 0.
__device__ __forceinline__ float clean(float x) { return x == x ? x + 0.f : -INFINITY; }
__device__ __forceinline__ float logit(const float* x, int i) { return clean(x[i]); }
__device__ __forceinline__ float logit(const uint16_t* x, int i) { return clean(bf16_bits_to_f32(x[i])); }

// Four logits from i on as they lie in memory (-inf past the end); rows are
// aligned to their type alone.
template <class T>
struct Raw;
template <>
struct Raw<float> {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ float low() { return -INFINITY; }
};
template <>
struct Raw<uint16_t> {
  typedef uint16_t vec __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ uint16_t low() { return 0xFF80; }
};
template <class T>
__device__ __forceinline__ typename Raw<T>::vec raw4(const T* x, int i, int end) {
  typename Raw<T>::vec v;
  if (i + 4 <= end) {
    v = *reinterpret_cast<const typename Raw<T>::vec*>(x + i);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = i + e < end ? x[i + e] : Raw<T>::low();
  }
  return v;
}
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(uint16_t v) { return bf16_bits_to_f32(v); }

// The tokens [from, to) of a workgroup of NT threads, kAhead vectors of four a
// thread and turn; the next turn's loads are on their way while one is worked
// on, and the first turn's from the constructor on.
constexpr int kAhead = 2;
template <class T, int NT>
struct Tokens {
  typename Raw<T>::vec v[kAhead];
  const T* x;
  int i, to;
  __device__ __forceinline__ Tokens(const T* row, int from, int end) : x(row), i(from + 4 * threadIdx.x), to(end) {
    load(v, i);
  }
  __device__ __forceinline__ void load(typename Raw<T>::vec (&d)[kAhead], int at) const {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) d[k] = raw4(x, min(at + 4 * NT * k, to), to);
  }
  template <class F>
  __device__ __forceinline__ void places(F f) {  // f(place in the thread's turn, logit)
    for (;;) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) f(4 * k + e, value(v[k][e]));
      i += 4 * NT * kAhead;
      if (i - 4 * (int)threadIdx.x >= to) break;
      load(v, i);
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F f) {  // f(token, logit, NaN and -0 as they are)
    for (; i < to; i += 4 * NT * kAhead) {
      typename Raw<T>::vec next[kAhead];
      load(next, i + 4 * NT * kAhead);
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) f(i + 4 * NT * k + e, value(v[k][e]));
#pragma unroll
      for (int k = 0; k < kAhead; ++k) v[k] = next[k];
    }
  }
};

// Order of logits as whole numbers, the largest logit first.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? b : ~b & 0x7FFFFFFFu;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k : ~k & 0x7FFFFFFFu);
}

constexpr float kLeast = -0x1.fffffep127f;  // the least finite logit

// A row's settings.
struct Row {
  float M;             // largest logit, 0 for a row with infinite ones
  bool inf;
  double c;            // log2(e) / T
  double floor_y;      // log2(min_p) (-inf: no floor)
  double top_p, u;
  int k, shift;
  float least;         // finite; tokens below it are not among the kept ones (or are -inf or NaN)
  int floor_bin;       // bin of the floor; kBins where there is none, kLast where it is past the range
  __device__ __forceinline__ void set_max(float largest);
  // Infinite logits take the whole weight: they become 0, finite ones so low
  // that they count and weigh nothing.
  __device__ __forceinline__ float seen(float x) const {
    return !inf || x == -INFINITY ? x : x == INFINITY ? 0.f : -0x1p127f;
  }
  // log2 of the weight.  It may lie far below all bins (a floor does so too:
  // min_p goes down to 2^-149), and weighs nothing from -64 on.
  __device__ __forceinline__ double y(float x) const { return ((double)x - (double)M) * c; }
  static __device__ __forceinline__ int bin(double y) { return min((int)(fmax(y, -64.0) * -(kLast / kRange)), kLast); }
  // 2^y 2^shift rounded to a whole number.  2^f, |f| <= 1/2: the polynomial of
  // degree 8 through its values at the Chebyshev nodes (off by 1.1e-12 at
  // most, exact at 0); adding 2^52 rounds to nearest and leaves the number in
  // the low bits.
  static __device__ __forceinline__ double exp2_of(double y, int up) {  // 2^(y + up)
    const double n = rint(y), t = y - n;
    double q = 1.3255224878668817e-06;
    q = fma(q, t, 1.5310079402249296e-05);
    q = fma(q, t, 0.00015403455852453838);
    q = fma(q, t, 0.0013333450568000645);
    q = fma(q, t, 0.009618129159402558);
    q = fma(q, t, 0.05550410941205933);
    q = fma(q, t, 0.2402265069581299);
    q = fma(q, t, 0.6931471805459335);
    q = fma(q, t, 1.0);
    return ldexp(q, (int)n + up);
  }
  __device__ __forceinline__ u64 weight(double y) const {
    return (u64)__double_as_longlong(exp2_of(y, shift) + 0x1p52) & 0x000FFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ u64 weight_of(float x) const {
    const double v = y(x);
    return bin(v) < kLast ? weight(v) : 0;
  }
  // A logit below which no token lies in the bins up to b: the bin's lower
  // edge, a few roundings lower.
  __device__ __forceinline__ float edge(int b) const {
    if (b >= kLast || inf || !(c > 0.0)) return kLeast;
    const float x = (float)((double)M - (b + 1.01) * (kRange / kLast) / c);
    return fmaxf(x - fabsf(x) * 0x1p-20f - 0x1p-100f, kLeast);
  }
};

struct Settings {
  float t, top_p, min_p, u;
  int k;
  __device__ __forceinline__ Settings(const SampleArgs& a, int r)
      : t(a.temperature ? a.temperature[r] : 1.f),
        top_p(a.top_p ? a.top_p[r] : 1.f),
        min_p(a.min_p ? a.min_p[r] : 0.f),
        u(a.u[r]),
        k(a.top_k ? a.top_k[r] : 0) {}
};

// What follows from the settings alone, asked for ahead of the largest logit.
__device__ __forceinline__ Row row_of(const SampleArgs& a, const Settings& set) {
  Row s;
  const bool greedy = !(set.t > 0.f);
  s.c = 1.4426950408889634 / (greedy ? 1.0 : (double)set.t);
  s.k = greedy ? 1 : set.k > 0 ? set.k : a.vocab;
  s.top_p = set.top_p < 1.f ? fmax((double)set.top_p, 0.0) : set.top_p >= 1.f ? 1.0 : 0.0;
  s.floor_y = set.min_p > 0.f ? log2((double)set.min_p) : -INFINITY;
  s.floor_bin = s.floor_y == -INFINITY ? kBins : Row::bin(fmin(s.floor_y, 0.0));
  s.u = set.u > 0.f ? fmin((double)set.u, 1.0 - 0x1p-24) : 0.0;
  s.shift = a.shift;
  return s;
}
__device__ __forceinline__ void Row::set_max(float largest) {
  inf = largest == INFINITY;
  M = inf ? 0.f : largest;
  if (inf) c = 1.4426950408889634;
  least = k == 1 ? largest : kLeast;
  if (floor_bin < kLast && top_p >= 1.0 && !inf) least = fmaxf(least, fminf(edge(floor_bin), M));
}

// ---- workgroup helpers of NT threads (every thread calls them)
// Reductions over the wave by DPP steps (rows of 16 lanes, then the last lanes
// of rows into the next ones): the result is in lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ float lane_f(float none, float v) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xF, false));
}
template <class F>
__device__ __forceinline__ float wave_join(float v, float none, F f) {
  v = f(v, lane_f<0x111, 0xF>(none, v));  // row_shr 1, 2, 4, 8
  v = f(v, lane_f<0x112, 0xF>(none, v));
  v = f(v, lane_f<0x114, 0xF>(none, v));
  v = f(v, lane_f<0x118, 0xF>(none, v));
  v = f(v, lane_f<0x142, 0xA>(none, v));  // row_bcast 15 into rows 1 and 3
  v = f(v, lane_f<0x143, 0xC>(none, v));  // row_bcast 31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_join(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_min(float v) {
  return wave_join(v, INFINITY, [](float a, float b) { return fminf(a, b); });
}
// The largest and the least finite value of the workgroup, and how many of
// its values are not -inf (PV a thread).
struct Spread {
  float M, low;
  uint32_t n;
};
template <int NT, int PV>
__device__ __forceinline__ Spread spread_of(const float (&v)[PV]) {
  __shared__ float sh[2][NT / 64];
  __shared__ uint32_t cnt[NT / 64];
  float M = -INFINITY, low = INFINITY;
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < PV; ++i) {
    const bool some = v[i] != -INFINITY;
    M = fmaxf(M, v[i]);
    low = some ? fminf(low, v[i]) : low;
    n += __popcll(__ballot(some));
  }
  M = wave_max(M);
  low = wave_min(low);
  if ((threadIdx.x & 63) == 0) {
    const int w = threadIdx.x >> 6;
    sh[0][w] = M, sh[1][w] = low, cnt[w] = n;
  }
  __syncthreads();
  Spread s{sh[0][0], sh[1][0], cnt[0]};
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) {
    s.M = fmaxf(s.M, sh[0][w]);
    s.low = fminf(s.low, sh[1][w]);
    s.n += cnt[w];
  }
  return s;
}

// One step of a scan over the wave: the value of the lane CTRL names (0 where
// there is none), in the rows of 16 lanes that ROWS has.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 from_lane(u64 v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_scan(u64 v) {
  v += from_lane<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += from_lane<0x112, 0xF>(v);
  v += from_lane<0x114, 0xF>(v);
  v += from_lane<0x118, 0xF>(v);
  v += from_lane<0x142, 0xA>(v);  // the last lane of the row before, into rows 1 and 3
  v += from_lane<0x143, 0xC>(v);  // lane 31, into rows 2 and 3
  return v;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_u(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += lane_u<0x111, 0xF>(v);
  v += lane_u<0x112, 0xF>(v);
  v += lane_u<0x114, 0xF>(v);
  v += lane_u<0x118, 0xF>(v);
  v += lane_u<0x142, 0xA>(v);
  v += lane_u<0x143, 0xC>(v);
  return v;
}
// Inclusive scans over the threads, of one value or of two; the totals go to all.
template <class U, int W>
struct Totals {
  U of[W];
  __device__ __forceinline__ void join(U& v, U& total, int wave) const {
    U before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const U x = of[w];
      if (w < wave) before += x;
      total += x;
    }
    v += before;
  }
};
template <int NT, class U>
__device__ __forceinline__ void block_scan(U& v, U& total) {
  __shared__ Totals<U, NT / 64> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) sh.of[wave] = v;
  __syncthreads();
  sh.join(v, total, wave);
}
template <int NT, class U, class V>
__device__ __forceinline__ void block_scan(U& u, U& total_u, V& v, V& total_v) {
  __shared__ Totals<U, NT / 64> sh_u;
  __shared__ Totals<V, NT / 64> sh_v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  u = wave_scan(u);
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) sh_u.of[wave] = u, sh_v.of[wave] = v;
  __syncthreads();
  sh_u.join(u, total_u, wave);
  sh_v.join(v, total_v, wave);
}

// ---- histogram of the tokens [from, to) into LDS, REP copies by lane; returns
// this thread's count of those above a floor past the range
template <class T, int NT, int REP>
__device__ __forceinline__ uint32_t count_tokens(Tokens<T, NT>& tokens, const Row& s, u64* w, uint32_t* c) {
  const int rep = threadIdx.x % REP;
  uint32_t over = 0, low = 0;
  const auto count = [&](float v) {
    const double y = s.y(v);
    const int b = Row::bin(y);
    if (s.floor_bin == kLast) over += y >= s.floor_y;
    if (b < kLast) {
      atomicAdd(&c[b * REP + rep], 1u);
      atomicAdd(&w[b * REP + rep], s.weight(y));
    } else {
      ++low;
    }
  };
  if (s.inf)
    tokens.each([&](int, float v) {
      if (v >= s.least) count(s.seen(v));
    });
  else
    tokens.each([&](int, float v) {
      if (v >= s.least) count(v);
    });
  if (low) atomicAdd(&c[kLast * REP + rep], low);
  return over;
}

// ---- where the places can lie
// Thread t holds the bins t PB .. t PB + PB - 1.
template <int NT>
struct Places {
  static constexpr int PB = kBins / NT;
  uint32_t c_at[PB], c_to[PB];  // before and after each bin
  u64 w_at[PB], w_to[PB];
  uint32_t live;
  u64 total;
  uint32_t k;
  uint32_t f_lo, f_hi;  // bounds of the count above the floor (equal: the count)
  uint32_t gathered;    // tokens of the bins that are needed
  int deepest;          // the last of them

  u64 w[PB];
  uint32_t c[PB];

  __device__ __forceinline__ void load(const u64* bin_w, const uint32_t* bin_c) {
#pragma unroll
    for (int i = 0; i < PB; ++i) w[i] = bin_w[threadIdx.x * PB + i], c[i] = bin_c[threadIdx.x * PB + i];
  }
  // `need` [kBins] gets 1 for the bins to gather.
  __device__ void find(const Row& s, uint32_t over_floor, uint8_t* need) {
    __shared__ u64 lohi[2];
    __shared__ uint32_t np[2];
    __shared__ int deep;
    if (threadIdx.x == 0) deep = 0;
    const int b0 = threadIdx.x * PB;
    uint32_t sum_c = 0;
    u64 sum_w = 0;
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      c_to[i] = sum_c += c[i];
      w_to[i] = sum_w += w[i];
      need[b0 + i] = 0;
    }
    const uint32_t own_c = sum_c;
    const u64 own_w = sum_w;
    block_scan<NT>(sum_c, live, sum_w, total);
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      c_to[i] += sum_c - own_c;
      w_to[i] += sum_w - own_w;
      c_at[i] = c_to[i] - c[i];
      w_at[i] = w_to[i] - w[i];
    }
    k = min((uint32_t)s.k, live);
    // Where a bin holds a place, the sum there is known to within the bin's
    // weight; the places that depend on it lie between the bins of the two
    // ends.  Nothing in the last bin weighs anything.
    const auto bounds = [&](uint32_t count, double& lo, double& hi) {  // weight at `count`
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PB; ++i)
        if (c_at[i] < count && count <= c_to[i]) {
          lohi[0] = count == c_to[i] ? w_to[i] : w_at[i];
          lohi[1] = w_to[i];
          if (count < c_to[i] && b0 + i < kLast) need[b0 + i] = 1;
        }
      __syncthreads();
      lo = (double)lohi[0];
      hi = (double)lohi[1];
    };
    if (s.floor_bin < kLast) {
#pragma unroll
      for (int i = 0; i < PB; ++i)
        if (b0 + i == s.floor_bin) {
          lohi[0] = c_at[i];
          lohi[1] = c_to[i];
          if (c_at[i] < c_to[i]) need[b0 + i] = 1;
        }
      __syncthreads();
      f_lo = max((uint32_t)lohi[0], 1u);
      f_hi = max((uint32_t)lohi[1], 1u);
    } else {
      f_lo = f_hi = s.floor_bin == kLast ? max(over_floor, 1u) : max(live, 1u);
    }
    double lo = 0, hi = 0;
    uint32_t n_lo = k, n_hi = k;  // bounds of the kept count
    if (s.top_p < 1.0) {
      bounds(k, lo, hi);
      lo *= s.top_p;
      hi *= s.top_p;
      if (threadIdx.x == 0) np[0] = 1, np[1] = hi > 0.0 ? k : 1;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        if (c_at[i] == c_to[i]) continue;
        const double at = (double)w_at[i], to = (double)w_to[i];
        if (to >= lo && at <= hi) need[b0 + i] = 1;
        if (to >= lo && at < lo) np[0] = c_at[i] + 1;
        if (to >= hi && at < hi) np[1] = c_to[i];
      }
      __syncthreads();
      n_lo = min(k, np[0]);
      n_hi = min(k, np[1]);
    }
    n_lo = min(n_lo, f_lo);
    n_hi = min(n_hi, f_hi);
    bounds(n_lo, lo, hi);
    const double d_lo = s.u * lo;
    if (n_hi != n_lo) bounds(n_hi, lo, hi);
    const double d_hi = s.u * hi;
    before = 0;
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if (c_at[i] < c_to[i] && (double)w_to[i] > d_lo && (double)w_at[i] <= d_hi) need[b0 + i] = 1;
      if (need[b0 + i]) {
        before += c_to[i] - c_at[i];
        atomicMax(&deep, b0 + i);
      }
    }
    block_scan<NT>(before, gathered);  // need[] and deep are complete behind it
    deepest = deep;
  }
  uint32_t before;  // gathered tokens up to and with this thread's bins
};

template <class T, int NT>
__device__ __forceinline__ void gather_tokens(Tokens<T, NT>& tokens, const Row& s, const uint8_t* need, float least,
                                              uint32_t* n, u64* cand) {
  tokens.each([&](int i, float v) {
    if (!(v >= least)) return;
    const float l = s.seen(clean(v));
    if (need[Row::bin(s.y(l))]) {
      const uint32_t at = atomicAdd(n, 1u);
      if (at < kGather) cand[at] = (u64)key_of(l) << 32 | (uint32_t)i;
    }
  });
}

struct Found {
  u64 count, weight;  // of the tokens before the value
  uint32_t key;       // the value
};

// The place of the row at which the running count or weight exceeds `target`,
// found digit by digit over the keys: four passes over the row.  For rows
// whose close bins hold more than fits (many equal logits, or flat ones).
template <class T, int NT>
__device__ Found radix_find(const T* x, int V, const Row& s, bool by_weight, u64 target, u64* hw, u64* hc) {
  static_assert(NT >= 256, "a digit a thread");
  __shared__ Found got;
  Found f{0, 0, 0};
  for (int level = 0; level < 4; ++level) {
    const int sft = 24 - 8 * level;
    __syncthreads();
    if (threadIdx.x < 256) hw[threadIdx.x] = hc[threadIdx.x] = 0;
    if (threadIdx.x == 0) got = f;
    __syncthreads();
    for (int i0 = 0; i0 < V; i0 += NT) {
      const int i = i0 + threadIdx.x;
      const float v = i < V ? s.seen(logit(x, i)) : -INFINITY;
      const uint32_t key = key_of(v);
      const bool in = v > -INFINITY && (s.inf || v >= s.least) && (level == 0 || (key >> (sft + 8)) == (f.key >> (sft + 8)));
      const int d = in ? (int)((key >> sft) & 255) : -1;
      u64 w = in ? s.weight_of(v) : 0;
      const u64 lanes = __ballot(in);
      if (!lanes) continue;
      // one digit in the whole wave (the usual case at the first levels): one
      // addition for it
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
    const u64 c = threadIdx.x < 256 ? hc[threadIdx.x] : 0, w = threadIdx.x < 256 ? hw[threadIdx.x] : 0;
    u64 to_c = c, to_w = w, all_c, all_w;
    block_scan<NT>(to_c, all_c, to_w, all_w);
    const u64 to = by_weight ? f.weight + to_w : f.count + to_c, at = to - (by_weight ? w : c);
    if (c > 0 && to > target && at <= target)
      got = Found{f.count + to_c - c, f.weight + to_w - w, f.key | (uint32_t)threadIdx.x << sft};
    __syncthreads();
    f = got;
  }
  return f;
}

// ---- the answers, by one workgroup
// N tokens in order with the running sums at them.
template <int N>
struct Ordered {
  u64 cand[N];         // (key, index)
  u64 run[N], w[N];    // the running weight, the token's own (before the sort: the tokens)
  uint32_t count[N];   // the running count
};
struct Digits {
  u64 w[256], c[256];
};

// The G tokens of m.w into m.cand, in order.  Up to a thread's worth each token
// counts those before it, shared out over the threads; more are sorted by
// exchanges (bitonic), of which those at a distance of up to 64 stay in the
// 128 tokens of a wave and need no barrier.  (A stage of exchanges is two
// dependent LDS round trips, 0.13 us: 100 tokens took 3.5 us so.)
template <int NT, int N>
__device__ __forceinline__ void sort_tokens(Ordered<N>& m, int G) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (G <= NT) {
    int pad = 64;
    while (pad < G) pad *= 2;
    const int i = tid % pad, part = tid / pad, parts = NT / pad;
    const u64 mine = i < G ? m.w[i] : 0;
    if (part == 0) m.count[i] = 0;
    __syncthreads();
    uint32_t rank = 0;
#pragma unroll 8
    for (int j = part; j < G; j += parts) rank += m.w[j] < mine;
    if (i < G && rank) atomicAdd(&m.count[i], rank);
    __syncthreads();
    if (part == 0 && i < G) m.cand[m.count[i]] = mine;
    __syncthreads();
    return;
  }
  int size = 2 * NT;
  while (size < G) size *= 2;
  for (int i = tid; i < size; i += NT) m.cand[i] = i < G ? m.w[i] : ~0ull;
  for (int len = 2, far = 1; len <= size; len *= 2)
    for (int j = len / 2; j > 0; j /= 2) {
      if (far || j > 64) __syncthreads();
      else __builtin_amdgcn_wave_barrier();
      far = j > 64;
      for (int i = tid; i < size / 2; i += NT) {
        const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
        const u64 p = m.cand[lo], q = m.cand[hi];
        if ((p > q) == ((lo & len) == 0)) m.cand[lo] = q, m.cand[hi] = p;
      }
    }
  __syncthreads();
}

__device__ __forceinline__ float logit_of(u64 cand) { return of_key((uint32_t)(cand >> 32)); }

__device__ __forceinline__ void write_answer(const SampleArgs& a, int r, const Row& s, int id, float best, u64 n, u64 W) {
  if (threadIdx.x != 0) return;
  a.ids[r] = id;
  if (a.prob) a.prob[r] = (float)(Row::exp2_of(s.y(best), s.shift) / (double)W);
  if (a.kept) a.kept[r] = (int32_t)n;
}

// The places, from G ordered tokens with their running sums; `end_of(count)`
// leaves in res[0] the sum at a count that is none of theirs.
template <int NT, int N, class E>
__device__ __forceinline__ void draw_from(const SampleArgs& a, int r, const Row& s, const Ordered<N>& m, int G, u64 k,
                                          u64 floor_n, u64* res, E end_of) {
  const int tid = threadIdx.x;
  const auto sum_at = [&](u64 count) -> u64 {
    end_of(count);
    __syncthreads();
    for (int i = tid; i < G; i += NT)
      if (m.count[i] == count) res[0] = m.run[i];
    __syncthreads();
    return res[0];
  };
  u64 n = min(k, floor_n);
  if (s.top_p < 1.0) {
    const double target = s.top_p * (double)sum_at(k);
    if (tid == 0) res[1] = target > 0.0 ? k : 1;
    __syncthreads();
    for (int i = tid; i < G; i += NT)
      if ((double)m.run[i] >= target && (double)(m.run[i] - m.w[i]) < target) res[1] = m.count[i];
    __syncthreads();
    n = min(n, res[1]);
  }
  const u64 W = sum_at(n);
  const double target = s.u * (double)W;
  if (tid == 0) res[2] = 0;
  __syncthreads();
  for (int i = tid; i < G; i += NT)
    if ((double)m.run[i] > target && (double)(m.run[i] - m.w[i]) <= target) res[2] = i;
  __syncthreads();
  const u64 drawn = m.cand[res[2]];
  write_answer(a, r, s, (int)(uint32_t)drawn, logit_of(drawn), n, W);
}

// The same from the row itself, by digits.  live, total: the tokens that are
// looked at and their weight; f_lo: their count above the floor where the bins
// do not leave it open.
template <class T, int NT>
__device__ void draw_by_digits(const SampleArgs& a, int r, const T* x, const Row& s, u64 live, u64 total, u64 k,
                               u64 floor_n, Digits& d) {
  __shared__ uint32_t over_s;
  __shared__ int at_s;
  const int tid = threadIdx.x, V = a.vocab;
  const auto find = [&](bool by_weight, u64 target) {
    return radix_find<T, NT>(x, V, s, by_weight, target, d.w, d.c);
  };
  const auto sum_at = [&](u64 count) -> u64 {
    if (count >= live) return total;
    const Found f = find(false, count - 1);
    return f.weight + (count - f.count) * s.weight_of(of_key(f.key));
  };
  __syncthreads();
  if (tid == 0) over_s = 0, at_s = 0;
  __syncthreads();
  if (s.floor_bin < kLast) {
    uint32_t over = 0;
    for (int i = tid; i < V; i += NT) {
      const float v = logit(x, i);
      over += v >= s.least && s.y(s.seen(v)) >= s.floor_y;
    }
    atomicAdd(&over_s, over);
    __syncthreads();
    floor_n = max(over_s, 1u);
  }
  u64 n = min(k, floor_n);
  if (s.top_p < 1.0) {
    const double target = s.top_p * (double)sum_at(k);
    u64 np = 1;
    if (target > 0.0) {
      // the first running weight >= target is the first > ceil(target) - 1
      const u64 t = (u64)ceil(target);
      const Found f = find(true, t - 1);
      const u64 w = max(s.weight_of(of_key(f.key)), 1ull);
      np = f.count + (t - f.weight + w - 1) / w;
    }
    n = min(n, np);
  }
  const u64 W = sum_at(n);
  const u64 t = (u64)floor(s.u * (double)W);
  const Found f = find(true, t);
  const float best = of_key(f.key);
  const u64 want = (t - f.weight) / max(s.weight_of(best), 1ull);  // this many equal ones come before it
  u64 seen = 0;
  for (int i0 = 0; i0 < V; i0 += NT) {
    const int i = i0 + tid;
    const bool eq = i < V && s.seen(logit(x, i)) == best;
    uint32_t to = eq, here;
    block_scan<NT>(to, here);
    if (eq && seen + to - 1 == want) at_s = i;
    seen += here;
    if (seen > want) break;
  }
  __syncthreads();
  write_answer(a, r, s, at_s, best, n, W);
}

// From the needed bins' tokens.
struct Answers {
  Ordered<kGather> m;
  uint8_t need[kBins];
  union {
    struct {
      u64 start[kBins], w_before[kBins];
      uint32_t first[kBins], c_before[kBins];
    } bin;
    Digits digits;
  };
  u64 res[3];
  uint32_t over;
};

template <class T>
__device__ void answer(const SampleArgs& a, int r, const T* x, const Row& s, const Places<kThreads>& pl, Answers& z) {
  constexpr int NT = kThreads, PB = Places<NT>::PB;
  const int tid = threadIdx.x, b0 = tid * PB;
  if (pl.gathered > kGather) {
    draw_by_digits<T, NT>(a, r, x, s, pl.live, pl.total, pl.k, pl.f_lo, z.digits);
    return;
  }
  auto& m = z.m;
  if (tid == 0) z.over = 0;
  const int G = (int)pl.gathered;
  {
    u64 at = pl.before;
#pragma unroll
    for (int i = PB - 1; i >= 0; --i) {
      if (z.need[b0 + i]) at -= pl.c_to[i] - pl.c_at[i];
      z.bin.first[b0 + i] = (uint32_t)at;
      z.bin.c_before[b0 + i] = (uint32_t)pl.c_at[i];
      z.bin.w_before[b0 + i] = pl.w_at[i];
    }
  }
  sort_tokens<NT>(m, G);
  // Running sums over the gathered tokens, `per` in a row a thread; taken off
  // where a bin begins, they are sums within the bin.
  const int per = (G + NT - 1) / NT, i0 = min(tid * per, G), i1 = min(i0 + per, G);
  u64 sum = 0, tot;
  uint32_t over = 0;
  for (int i = i0; i < i1; ++i) {
    const double y = s.y(logit_of(m.cand[i]));
    const int b = Row::bin(y);
    const u64 w = b < kLast ? s.weight(y) : 0;
    sum += w;
    m.w[i] = w;
    over += b == s.floor_bin && y >= s.floor_y;
  }
  if (over) atomicAdd(&z.over, over);
  const u64 own = sum;
  block_scan<NT>(sum, tot);
  u64 at = sum - own;
  for (int i = i0; i < i1; ++i) {
    const int b = Row::bin(s.y(logit_of(m.cand[i])));
    if ((uint32_t)i == z.bin.first[b]) z.bin.start[b] = at;
    at += m.w[i];
    m.run[i] = at;
  }
  __syncthreads();
  for (int i = i0; i < i1; ++i) {  // in the whole row
    const int b = Row::bin(s.y(logit_of(m.cand[i])));
    m.run[i] += z.bin.w_before[b] - z.bin.start[b];
    m.count[i] = z.bin.c_before[b] + (i - z.bin.first[b]) + 1;
  }
  const u64 floor_n = s.floor_bin < kLast ? max((u64)z.bin.c_before[s.floor_bin] + z.over, 1ull) : pl.f_lo;
  __syncthreads();
  draw_from<NT>(a, r, s, m, G, pl.k, floor_n, z.res, [&](u64 count) {
#pragma unroll
    for (int i = 0; i < PB; ++i)  // a bin's end, or nothing more weighs anything
      if (pl.c_at[i] < count && count <= pl.c_to[i]) z.res[0] = pl.w_to[i];
  });
}

// From the G likeliest tokens of the row (all that can be kept among them), in
// any order in m.w.
template <int NT>
__device__ __forceinline__ void answer_flat(const SampleArgs& a, int r, const Row& s, Ordered<kFlat>& m, int G, u64* res) {
  const int tid = threadIdx.x;
  sort_tokens<NT>(m, G);
  const int per = (G + NT - 1) / NT, i0 = min(tid * per, G), i1 = min(i0 + per, G);
  u64 sum = 0, tot;
  uint32_t over = 0, above;
  for (int i = i0; i < i1; ++i) {
    const double y = s.y(logit_of(m.cand[i]));
    const u64 w = Row::bin(y) < kLast ? s.weight(y) : 0;
    sum += w;
    over += y >= s.floor_y;
    m.w[i] = w;
  }
  const u64 own = sum;
  block_scan<NT>(over, above, sum, tot);
  u64 at = sum - own;
  for (int i = i0; i < i1; ++i) {
    at += m.w[i];
    m.run[i] = at;
    m.count[i] = i + 1;
  }
  __syncthreads();
  draw_from<NT>(a, r, s, m, G, min((u64)s.k, (u64)G), max(above, 1u), res, [](u64) {});
}

// A bound that at least k of the values (PV a thread, -inf for none) reach,
// close to the k-th largest: 256 steps from the largest down to the least,
// counted.  kLeast where there are fewer than k.
template <int NT, int PV>
__device__ __forceinline__ float kth_bound(const float (&v)[PV], const Spread& of, int k) {
  __shared__ uint32_t steps[256];
  __shared__ int at_s;
  const int tid = threadIdx.x;
  if (of.n < (uint32_t)k) return kLeast;
  if (k == 1) return of.M;
  const float step = (of.M - of.low) * (1.f / 255.f);
  if (!(step > 0.f && step < INFINITY)) return fmaxf(of.low, kLeast);  // all equal, or too far apart for float
  if (tid < 256) steps[tid] = 0;
  if (tid == 0) at_s = 255;
  __syncthreads();
  const float scale = 1.f / step;
#pragma unroll
  for (int i = 0; i < PV; ++i)
    if (v[i] != -INFINITY) atomicAdd(&steps[min((int)((of.M - v[i]) * scale), 255)], 1u);
  __syncthreads();
  if (tid < 64) {  // one wave: four steps a lane
    uint32_t c[4], n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += c[i] = steps[4 * tid + i];
    uint32_t to = (uint32_t)wave_scan(n) - n;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (to < (uint32_t)k && to + c[i] >= (uint32_t)k) at_s = 4 * tid + i;
      to += c[i];
    }
  }
  __syncthreads();
  // the step's lower end, a few roundings lower
  const float x = of.M - (at_s + 1.01f) * step;
  return fmaxf(x - fabsf(x) * 0x1p-20f - fabsf(of.M) * 0x1p-20f, of.low);
}

// Tokens that reach `least` are added to m.w as they are found: a thread looks
// through its turn of tokens, then takes places for all it keeps at once.
struct Keep {
  uint32_t* n;
  u64* w;
  float least;
  template <int B, class V>
  __device__ __forceinline__ void operator()(const Row& s, const V (&raw)[B], const int (&at)[B]) const {
    uint32_t mask = 0;
#pragma unroll
    for (int e = 0; e < B; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) mask |= (uint32_t)(value(raw[e][k]) >= least) << (4 * e + k);
    if (!mask) return;
    uint32_t to = atomicAdd(n, (uint32_t)__popc(mask));
#pragma unroll
    for (int e = 0; e < B; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (mask >> (4 * e + k) & 1) {
          if (to < kFlat) w[to] = (u64)key_of(s.seen(clean(value(raw[e][k])))) << 32 | (uint32_t)(at[e] + k);
          ++to;
        }
  }
};

// Rows of nothing that can be drawn.
__device__ __forceinline__ bool empty_row(const SampleArgs& a, int r, float M) {
  if (M != -INFINITY) return false;
  if (threadIdx.x == 0) {
    a.ids[r] = -1;
    if (a.prob) a.prob[r] = 0.f;
    if (a.kept) a.kept[r] = 0;
  }
  return true;
}

template <class T>
__device__ __forceinline__ const T* row_ptr(const SampleArgs& a, int r) {
  return (const T*)a.logits + (long long)r * a.ld;
}

// A row of up to kOneBlock tokens.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a) {
  constexpr int NT = kThreads;
  __shared__ union {
    struct {
      u64 w[kBins];
      uint32_t c[kBins];
    } bins;
    Ordered<kFlat> flat;
  } h;
  __shared__ Answers z;
  __shared__ uint32_t n_cand, over;
  const int r = blockIdx.x, V = a.vocab;
  const T* x = row_ptr<T>(a, r);
  const Settings set(a, r);
  Tokens<T, NT> first(x, 0, V), again = first, last = first;  // the first turn is loaded once
  Row s = row_of(a, set);
  // The tokens in one place of the turns are a group: each token its own up to
  // 4096 of them, and top-k's bound leaves hardly more than k.
  constexpr int PV = 4 * kAhead;
  float group[PV];
#pragma unroll
  for (int e = 0; e < PV; ++e) group[e] = -INFINITY;
  first.places([&](int e, float v) { group[e] = fmaxf(group[e], v); });  // of a number and NaN the number
  if (threadIdx.x == 0) n_cand = over = 0;
  const Spread of = spread_of<NT, PV>(group);
  if (empty_row(a, r, of.M)) return;
  s.set_max(of.M);
  // Few tokens, or top-k by the groups.
  if (V <= NT || (uint32_t)s.k <= min(of.n, (uint32_t)kFlatK)) {
    const float bound = V <= NT ? kLeast : kth_bound<NT, PV>(group, of, s.k);
    const Keep keep{&n_cand, h.flat.w, bound};
    for (int i0 = 0;;) {
      int at[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) at[k] = again.i + 4 * NT * k;
      keep(s, again.v, at);
      again.i += 4 * NT * kAhead;
      if ((i0 += 4 * NT * kAhead) >= V) break;
      again.load(again.v, again.i);
    }
    __syncthreads();
    if (n_cand <= kFlat) {
      answer_flat<NT>(a, r, s, h.flat, n_cand, z.res);
      return;
    }
    again = last;
    __syncthreads();  // every thread has read n_cand
  }
  for (int i = threadIdx.x; i < kBins; i += NT) h.bins.w[i] = 0, h.bins.c[i] = 0;
  if (threadIdx.x == 0) n_cand = 0;
  __syncthreads();
  const uint32_t ov = count_tokens<T, NT, 1>(again, s, h.bins.w, h.bins.c);
  if (ov) atomicAdd(&over, ov);
  __syncthreads();
  Places<NT> pl;
  pl.load(h.bins.w, h.bins.c);
  pl.find(s, over, z.need);
  if (pl.gathered <= kGather)
    gather_tokens<T, NT>(last, s, z.need, fmaxf(s.least, s.edge(pl.deepest)), &n_cand, z.m.w);
  answer<T>(a, r, x, s, pl, z);
}

// ---- long rows.  Each kernel asks for all that it reads first.
// Group q of a row: the tokens of `lanes` neighbouring threads of a chunk.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_max_kernel(SampleArgs a) {
  const int r = blockIdx.y, ch = blockIdx.x;
  RowWork& wk = a.work[r];
  Tokens<T, kThreads> tokens(row_ptr<T>(a, r), ch * a.chunk, min((ch + 1) * a.chunk, a.vocab));
  for (int b = ch * kThreads + threadIdx.x; b < kBins; b += a.chunks * kThreads) wk.w[b] = 0, wk.c[b] = 0;
  if (ch == 0 && threadIdx.x == 0) wk.gathered = wk.over_floor = 0;
  float M = -INFINITY;
  tokens.each([&](int, float v) { M = fmaxf(M, v); });  // of a number and NaN the number
  for (int off = 1; off < a.lanes; off *= 2) M = fmaxf(M, shfl_xor_f(M, off));
  const int g = (ch * kThreads + threadIdx.x) / a.lanes;
  if (threadIdx.x % a.lanes == 0 && g < kGroups) wk.group_max[g] = M;
}

// The groups' largest logits, kGroups / NT a thread, and the row's.
template <int NT>
struct Groups {
  static constexpr int PV = kGroups / NT;
  float v[PV];
  __device__ __forceinline__ Groups(const SampleArgs& a, const RowWork& wk) {
    const int n = min(a.chunks * (kThreads / a.lanes), kGroups);
#pragma unroll
    for (int i = 0; i < PV; ++i) {
      const int g = i * NT + threadIdx.x;
      v[i] = g < n ? wk.group_max[g] : -INFINITY;
    }
  }
};

// Whether the row goes by its groups: by its settings alone.
__device__ __forceinline__ bool by_groups(const SampleArgs& a, const Row& s) {
  return s.k <= min(kFlatK, a.chunks * (kThreads / a.lanes));
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_count_kernel(SampleArgs a) {
  __shared__ u64 hw[kBins * kReplicas];
  __shared__ uint32_t hc[kBins * kReplicas];
  const int r = blockIdx.y, ch = blockIdx.x, tid = threadIdx.x;
  RowWork& wk = a.work[r];
  const Settings set(a, r);
  const Groups<kThreads> gr(a, wk);
  Tokens<T, kThreads> tokens(row_ptr<T>(a, r), ch * a.chunk, min((ch + 1) * a.chunk, a.vocab));
  Row s = row_of(a, set);
  if (by_groups(a, s)) return;
  const float M = spread_of<kThreads>(gr.v).M;
  if (M == -INFINITY) return;
  s.set_max(M);
  for (int i = tid; i < kBins * kReplicas; i += kThreads) hw[i] = 0, hc[i] = 0;
  __syncthreads();
  uint32_t over = count_tokens<T, kThreads, kReplicas>(tokens, s, hw, hc);
  if (s.floor_bin == kLast) {
    for (int off = 32; off > 0; off >>= 1) over += __shfl_xor(over, off, 64);
    if ((tid & 63) == 0) atomicAdd(&wk.over_floor, over);
  }
  __syncthreads();
  for (int b = tid; b < kBins; b += kThreads) {
    u64 w = 0;
    uint32_t c = 0;
#pragma unroll
    for (int k = 0; k < kReplicas; ++k) w += hw[b * kReplicas + k], c += hc[b * kReplicas + k];
    if (c) {
      atomicAdd(&wk.c[b], c);
      if (w) atomicAdd(&wk.w[b], w);
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_gather_kernel(SampleArgs a) {
  __shared__ uint8_t need[kBins];
  __shared__ u64 cand[kGather];
  __shared__ uint32_t n, base;
  const int r = blockIdx.y, ch = blockIdx.x;
  RowWork& wk = a.work[r];
  const Settings set(a, r);
  const Groups<kThreads> gr(a, wk);
  Places<kThreads> pl;
  pl.load(wk.w, wk.c);
  const uint32_t over = wk.over_floor;
  Tokens<T, kThreads> tokens(row_ptr<T>(a, r), ch * a.chunk, min((ch + 1) * a.chunk, a.vocab));
  if (threadIdx.x == 0) n = 0;
  Row s = row_of(a, set);
  if (by_groups(a, s)) return;
  const float M = spread_of<kThreads>(gr.v).M;
  if (M == -INFINITY) return;
  s.set_max(M);
  pl.find(s, over, need);
  if (pl.gathered > kGather) return;
  gather_tokens<T, kThreads>(tokens, s, need, fmaxf(s.least, s.edge(pl.deepest)), &n, cand);
  __syncthreads();
  if (threadIdx.x == 0 && n) base = atomicAdd(&wk.gathered, n);
  __syncthreads();
  for (int i = threadIdx.x; i < (int)n && base + i < kGather; i += kThreads) wk.cand[base + i] = cand[i];
}

// A row that goes by its groups.
template <class T>
__device__ __forceinline__ void answer_by_groups(const SampleArgs& a, int r, const T* x, Row s, const Spread& of,
                                                 const Groups<kThreads>& gr, Ordered<kFlat>& m, Digits& digits,
                                                 int* list, uint32_t* n_list, uint32_t* n_cand, u64* res) {
  constexpr int PV = Groups<kThreads>::PV;
  const int tid = threadIdx.x;
  const float least = kth_bound<kThreads, PV>(gr.v, of, s.k);
  // the listed groups' first tokens (a chunk is a whole number of turns)
  const int log_lanes = __builtin_ctz(a.lanes), log_groups = __builtin_ctz(kThreads / a.lanes);
  uint32_t reach = 0;
#pragma unroll
  for (int i = 0; i < PV; ++i) reach += gr.v[i] >= least;
  if (reach) {
    uint32_t to = atomicAdd(n_list, reach);
#pragma unroll
    for (int i = 0; i < PV; ++i)
      if (gr.v[i] >= least) {
        const int g = i * kThreads + tid;
        list[to++] = (g >> log_groups) * a.chunk + 4 * ((g << log_lanes) & (kThreads - 1));
      }
  }
  __syncthreads();
  // Their vectors of four tokens, turn by turn, kBatch loads of a thread at once.
  constexpr int kBatch = 4;
  const Keep keep{n_cand, m.w, least};
  const int width = (int)*n_list << log_lanes, n = width * (a.chunk / (4 * kThreads));
  const uint32_t inv = width > 1 ? (uint32_t)(((1ull << 32) + width - 1) / (unsigned)width) : 0u;
  for (int v0 = tid; v0 < n; v0 += kBatch * kThreads) {
    typename Raw<T>::vec raw[kBatch];
    int at[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const int v = min(v0 + e * kThreads, n - 1);
      int turn = inv ? (int)__umulhi((uint32_t)v, inv) : v;  // v / width, at most one more
      turn -= turn * width > v;
      const int q = v - turn * width;
      at[e] = v == v0 + e * kThreads ? list[q >> log_lanes] + 4 * ((q & (a.lanes - 1)) + kThreads * turn) : a.vocab;
      raw[e] = raw4(x, min(at[e], a.vocab), a.vocab);
    }
    keep(s, raw, at);
  }
  __syncthreads();
  const uint32_t G = *n_cand;
  if (G <= kFlat) {
    answer_flat<kThreads>(a, r, s, m, (int)G, res);
    return;
  }
  // very many equal logits: from the whole row, past the groups' bound
  s.least = s.inf ? kLeast : least;
  u64 sum = 0, total;
  uint32_t live_n = 0, live, over = 0, above;
  Tokens<T, kThreads> tokens(x, 0, a.vocab);
  tokens.each([&](int, float v) {
    if (!(v >= s.least)) return;
    const double y = s.y(s.seen(v));
    ++live_n;
    sum += Row::bin(y) < kLast ? s.weight(y) : 0;
    over += y >= s.floor_y;
  });
  block_scan<kThreads>(live_n, live, sum, total);
  block_scan<kThreads>(over, above);
  draw_by_digits<T, kThreads>(a, r, x, s, live, total, min((uint32_t)s.k, live), max(above, 1u), digits);
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_answer_kernel(SampleArgs a) {
  __shared__ union {
    Answers z;
    struct {
      Ordered<kFlat> m;
      Digits digits;
      int list[kGroups];
    } flat;
  } h;
  __shared__ uint32_t n_list, n_cand;
  __shared__ u64 res[3];
  const int r = blockIdx.x;
  RowWork& wk = a.work[r];
  const T* x = row_ptr<T>(a, r);
  const Settings set(a, r);
  const Groups<kThreads> gr(a, wk);
  Places<kThreads> pl;
  pl.load(wk.w, wk.c);
  const uint32_t over = wk.over_floor;
  const u64 mine = wk.cand[threadIdx.x];
  if (threadIdx.x == 0) n_list = n_cand = 0;
  Row s = row_of(a, set);
  const Spread of = spread_of<kThreads>(gr.v);
  if (empty_row(a, r, of.M)) return;
  s.set_max(of.M);
  if (by_groups(a, s)) {
    answer_by_groups<T>(a, r, x, s, of, gr, h.flat.m, h.flat.digits, h.flat.list, &n_list, &n_cand, res);
    return;
  }
  pl.find(s, over, h.z.need);
  if (pl.gathered <= kGather) {
    h.z.m.w[threadIdx.x] = mine;
    for (int i = threadIdx.x + kThreads; i < (int)pl.gathered; i += kThreads) h.z.m.w[i] = wk.cand[i];
  }
  answer<T>(a, r, x, s, pl, h.z);
}

template <class T>
void launch(const SampleArgs& a, int n_rows, hipStream_t st) {
  if (a.vocab <= kOneBlock) {
    sample_row_kernel<T><<<n_rows, kThreads, 0, st>>>(a);
    return;
  }
  const dim3 grid(a.chunks, n_rows);
  sample_max_kernel<T><<<grid, kThreads, 0, st>>>(a);
  sample_count_kernel<T><<<grid, kThreads, 0, st>>>(a);
  sample_gather_kernel<T><<<grid, kThreads, 0, st>>>(a);
  sample_answer_kernel<T><<<n_rows, kThreads, 0, st>>>(a);
}

}  // namespace
}  // namespace ooo

using namespace ooo;

extern "C" size_t ooo_sample_workspace(int32_t n_rows, int32_t vocab) {
  if (n_rows < 1 || vocab < 1 || vocab > (1 << 20)) return 0;
  return vocab <= kOneBlock ? 16 : (size_t)n_rows * sizeof(RowWork);
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
  OOO_REQUIRE(n_rows <= 65535, OOO_ERR_UNSUPPORTED, "ooo_sample: n_rows %d above 65535", n_rows);
  OOO_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 15) == 0, OOO_ERR_UNSUPPORTED,
              "ooo_sample: workspace is not 16-byte aligned");
  OOO_REQUIRE(ws_bytes >= ooo_sample_workspace(n_rows, vocab), OOO_ERR_CAPACITY,
              "ooo_sample: workspace of %zu bytes needed (got %zu)", ooo_sample_workspace(n_rows, vocab), ws_bytes);
  int log2v = 0;
  while ((1 << log2v) < vocab) ++log2v;
  // sums stay below 2^63, weights below 2^51 (see Row::weight)
  const int shift = 62 - log2v < 50 ? 62 - log2v : 50;
  SampleArgs a{logits, ld, vocab, shift, temperature, top_k, top_p, min_p, u, ids, prob, kept, (RowWork*)workspace, 0, 0, 1};
  // About eight workgroups a CU, of at least 4096 tokens (two loads of 16 bytes
  // a thread): the rows that are counted are few among those that are not, and
  // have to spread.
  const int most = (vocab + 4095) / 4096, want = (8 * device_cus() + n_rows - 1) / n_rows;
  const int chunks = want < most ? want : most;
  a.chunk = ((vocab + chunks - 1) / chunks + 2047) / 2048 * 2048;
  a.chunks = (vocab + a.chunk - 1) / a.chunk;
  a.lanes = 1;
  while (a.chunks * (kThreads / a.lanes) > kGroups) a.lanes *= 2;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dt == OOO_BF16) launch<uint16_t>(a, n_rows, st);
  else launch<float>(a, n_rows, st);
  const hipError_t e = hipGetLastError();
  OOO_REQUIRE(e == hipSuccess, OOO_ERR_HIP, "ooo_sample: launch failed: %s", hipGetErrorString(e));
  return ooo::ok();
}
