// The next token of every row of logits, from a given random number: temperature, top-k, top-p, min-p.
//
//   w_i = exp((x_i - max) / T); order: larger x first, of equal ones the lower index.  S1: the first k.  S2: those of S1 before which less
//   than p of S1's mass lies.  S3: those with w_i >= min_p.  kept = S1, S2 and S3, at least the first; the token is the first kept one in
//   index order at which the running sum of the kept weights exceeds u times their total.
//
// All three filters cut the order at one place, so the work is to find that place without sorting.
//   * A row belongs to a cluster of up to 8 CTAs.  Its logits come from HBM once: the rows that are worked on stay in L2, and what a pass needs
//     again is read from there.  What the CTAs have to agree on goes through distributed shared memory.
//   * Weights are fixed-point numbers of 43 bits behind the point, from exponentials in double: their sums are whole numbers, the same in
//     any order, and a border between two tokens of a hundred thousand falls where 64-bit arithmetic puts it (float32 sums of such a
//     row are off by as much as a token's weight).
//   * In the first pass every thread keeps the maximum of each 4 pieces of 16 bytes that it looks at.  A histogram of these maxima says from
//     which value on there are at least k elements (as many groups have one); the few elements above it are gathered, nearly all
//     groups unseen, and one CTA finishes on the list.  Top-p does the same with two such values, if what lies above one of them has enough mass.
//   * Where what is kept does not fit into a list, passes that sum mass and count above several values at once narrow the place of the cut
//     down until its neighbourhood fits; equal logits by the thousand are cut by index.  The kept weights are then summed by warps over
//     contiguous ranges, and only the range that the random number falls into is walked.
// Bound by latency for few rows: a greedy row of 131072 takes 5.5 us, one with a few candidates 11 - 14 (three cluster barriers, as all
// rows that end on their first list or keep everything, and some 14 of the block, the last of them in one CTA alone), one that keeps thousands
// 27 - 44 (seven to nine cluster barriers and three or four passes from L2 of 4 - 10 us each).  256 x 150001 float32: greedy 46 us,
// 3.4 TB/s, as the first pass of a row and the steps behind it do not overlap within its cluster; top-k 65, unfiltered 97, top-p 204.
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include <cuda_bf16.h>

#include "mq_common.cuh"
#include "mq_sample_order.h"

namespace mq {
namespace {

// (a step that the compiler makes a call of has its operands in local memory, and takes four times as long)
#define MQ_INLINE __attribute__((always_inline))

constexpr int kThreads = 256, kWarps = kThreads / 32;
// CTAs to an SM.  float32: 256 x 150001, top-k 50: 66 us, 76 with 3.  bf16, whose pieces are twice as many elements in registers: 64 x 131072
// with filters as in use 67 us, 72 with 4; 1 x 131072, greedy, 6.8 us, 7.9 with 4 (256 x 150001 loses by it: 175 us, 168 with 4; an earlier form's times)
template <typename T>
constexpr int kCtas = sizeof(T) == 4 ? 4 : 3;
constexpr int kCap = 2048;            // candidates of a list
constexpr int kMaxCluster = 8;
constexpr int kGroup = 4;             // pieces of 16 bytes whose maximum is kept
constexpr int kBars = 1024;           // bars of a histogram: of these, eight to a unit, from -64 on; of all elements, 32 to a unit, up to the maximum's
constexpr int kPairs = 256;           // a list of up to so many is compared pair by pair
constexpr int kShort = 160;           // candidates that a nucleus is looked for in first
constexpr int kLong = 1280;           // the largest k that the groups' bars serve
constexpr int kEdges = 2;             // values that a narrowing pass sums above
constexpr int kLevels = 32;           // more than a narrowing takes: a bound, so that no rows whatever can keep a kernel in it
constexpr int kItems = 2 * kEdges > kWarps + 1 ? 2 * kEdges : kWarps + 1;   // what a CTA tells the others at once
constexpr int kPoint = 43;            // bits behind the point of a weight: 2^20 of them stay below 2^63
constexpr int kMaxVocab = 1 << 20;
constexpr int kTable = 1024;          // 2^(j / kTable)
constexpr int kListBytes = 2 * kCap * 8;
constexpr int kMaximaMost = (kMaxVocab / kMaxCluster / 4 + kThreads * kGroup) / kGroup * 4;

struct SampleArgs {
  const void* x;
  int64_t ld;
  int V, per;          // columns, and those of a CTA
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* token;
  float* logp;
  int32_t* kept;
};

// Floats (no NaN; -0 as 0) in their order as whole numbers, and back
__device__ __forceinline__ uint32_t order_key(float x) { return order_of_bits(__float_as_uint(x)); }
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(bits_of_order(k)); }
// floor(x * 2^23 / 2^e) for a small |x|: the sum with 1.5 * 2^e, rounded down, has it in its low bits
__device__ __forceinline__ int floor_bits(float x, float magic) { return (int)(__float_as_uint(__fadd_rd(x, magic)) - __float_as_uint(magic)); }
// floor(8 x) + 512, at most the last bar (x >= -64); floor(32 x)
__device__ __forceinline__ int bar_of(float x) { return floor_bits(fminf(x, 63.875f), 1572864.0f) + kBars / 2; }
__device__ __forceinline__ int fine_of(float x) { return floor_bits(fminf(x, 63.96875f), 393216.0f); }

// An entry of a list: the key of a logit (16 bits say it of a bf16 number), then the index, downwards.  As many bits as can differ: a list is
// searched by 8 of them at a time.
constexpr int kIndexBits = 20;
constexpr uint32_t kIndexMask = (1u << kIndexBits) - 1u;
template <typename T>
__device__ __forceinline__ uint64_t entry_of(float x, int i) {
  return (uint64_t)(order_key(x) >> (sizeof(T) == 2 ? 16 : 0)) << kIndexBits | ((uint32_t)~i & kIndexMask);
}
__device__ __forceinline__ int entry_index(uint64_t e) { return (int)(~(uint32_t)e & kIndexMask); }
template <typename T>
__device__ __forceinline__ float entry_value(uint64_t e) {
  const uint32_t k = (uint32_t)(e >> kIndexBits);
  return key_value(sizeof(T) == 4 ? k : k << 16);
}
// the first entry whose value is not below x
template <typename T>
__device__ __forceinline__ uint64_t first_entry(float x) {
  const uint32_t k = order_key(x);
  return (uint64_t)(sizeof(T) == 4 ? k : (k + 0xffffu) >> 16) << kIndexBits;
}

// The larger one; NaN if one of them is
__device__ __forceinline__ float max_or_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// what stands in the place of `mine` in another CTA of the cluster
template <typename T>
__device__ __forceinline__ T peer_load(const T* mine, uint32_t rank) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(mine)), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  if (sizeof(T) == 8) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(r) : "memory");
    return (T)v;
  }
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
  return (T)v;
}

__device__ __forceinline__ uint4 peer_load4(const uint32_t* mine, uint32_t rank) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(mine)), r;
  uint4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(r) : "memory");
  return v;
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Where the order is cut: larger elements are kept, and of those equal to `value` the ones up to column idx
struct Cut {
  float value;
  int idx;
  __device__ __forceinline__ bool keeps(float x, int i) const { return x > value || (x == value && i <= idx); }
};

template <typename T>
struct Row {
  static constexpr int kE = 16 / (int)sizeof(T);   // elements of a 16-byte piece
  const T* x;          // the row
  float* maxima;       // [group][thread] of this thread's pieces
  int i0, i1;          // columns of this CTA
  int lead;            // elements of the first piece in front of column i0
  int pieces;
  int w0, wn;          // pieces w0 .. w0 + wn - 1 have no other columns
  bool odd;            // the row has a NaN or +infinity somewhere

  __device__ __forceinline__ float widen(T v) const;
  // NaN: never; +infinity is the largest number of the type
  static constexpr float kMost = sizeof(T) == 4 ? FLT_MAX : 3.3895313892515355e38f;
  __device__ __forceinline__ static float clean(float v) { return v == v ? fminf(v, kMost) : -INFINITY; }

  // columns i0 - lead + kE v ..; those that are not this CTA's read as -inf
  __device__ __forceinline__ void global(int v, float (&out)[kE]) const {
    const int first = i0 - lead + v * kE;
    if ((unsigned)(v - w0) < (unsigned)wn) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(x + first));
      unpack(q, out);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) out[e] = first + e >= i0 && first + e < i1 ? widen(x[first + e]) : -INFINITY;
    }
  }
  __device__ __forceinline__ void unpack(const uint4& q, float (&out)[kE]) const;
  // the same in its own bits
  __device__ __forceinline__ uint32_t bits_of(int i) const;
  __device__ __forceinline__ uint4 raw(int v) const {
    const int first = i0 - lead + v * kE;
    if ((unsigned)(v - w0) < (unsigned)wn) return __ldg(reinterpret_cast<const uint4*>(x + first));
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = sizeof(T) == 4 ? bits_of(first + e) : bits_of(first + 2 * e) | bits_of(first + 2 * e + 1) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ int column(int v) const { return i0 - lead + v * kE; }
  __device__ __forceinline__ void get(int v, float (&out)[kE]) const {
    global(v, out);
    if (odd) {
#pragma unroll
      for (int e = 0; e < kE; ++e) out[e] = clean(out[e]);
    }
  }
};
template <>
__device__ __forceinline__ float Row<float>::widen(float v) const { return v; }
template <>
__device__ __forceinline__ uint32_t Row<float>::bits_of(int i) const { return i >= i0 && i < i1 ? __float_as_uint(x[i]) : 0xff800000u; }
template <>
__device__ __forceinline__ uint32_t Row<__nv_bfloat16>::bits_of(int i) const {
  return i >= i0 && i < i1 ? (uint32_t)__bfloat16_as_ushort(x[i]) : 0xff80u;
}
template <>
__device__ __forceinline__ void Row<float>::unpack(const uint4& q, float (&out)[4]) const {
  out[0] = __uint_as_float(q.x); out[1] = __uint_as_float(q.y); out[2] = __uint_as_float(q.z); out[3] = __uint_as_float(q.w);
}
template <>
__device__ __forceinline__ float Row<__nv_bfloat16>::widen(__nv_bfloat16 v) const { return __bfloat162float(v); }
template <>
__device__ __forceinline__ void Row<__nv_bfloat16>::unpack(const uint4& q, float (&out)[8]) const {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    out[2 * e] = __uint_as_float(w[e] << 16);
    out[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
// exp((x - m) / T) as a fixed-point number: 2^(d c) = 2^r 2^f with r = d c rounded to multiples of 1 / kTable, 2^r from a table and
// the exponent's bits, 2^f by the exponential's series (the first term left out is below 2^-37 of the sum, and as often above as below 0).  The sum with 512 leaves the rounded number in the low bits of a
// double whose upper bits are always the same: sums over such patterns are sums of weights once these bits are taken off, once per
// term.  No branches, so that the chains of several elements overlap; what is far down is lifted to `low`, whose weight rounds to 0.
constexpr uint64_t kBias = 0x4080000000000000ull;   // the bits of 512.0
struct Weight {
  double m, c;            // c = log2(e) / T
  float low;
  const double* table;
  __device__ __forceinline__ uint64_t biased(float x) const {
    const double d = (double)fmaxf(x, low) - m;            // <= 0
    const double magic = 6755399441055744.0 / kTable;      // 1.5 * 2^52 / kTable: adding it rounds to multiples of 1 / kTable
    const double a = fma(d, c, magic);
    const double f = fma(d, c, magic - a);
    const int n = (int)(uint32_t)__double_as_longlong(a);  // round(d c kTable), in the low bits
    const double p = fma(fma(f, 2.402265069591007123e-1, 6.931471805599453094e-1), f, 1.0);   // ln(2)^k / k!
    const double s = table[n & (kTable - 1)];
    const double scaled = __hiloint2double(__double2hiint(s) + ((n & ~(kTable - 1)) << 10), __double2loint(s));
    return (uint64_t)__double_as_longlong(fma(scaled, p, 512.0));
  }
  __device__ __forceinline__ uint64_t operator()(float x) const { return biased(x) - kBias; }
};
static_assert(kPoint == 43 && kTable == 1024, "512 = 2^(52 - kPoint); 2^10 = 2^20 / kTable");

template <typename Tx>
struct Smem {
  uint64_t exch[2][kItems];             // what the others fetch
  uint64_t warp_part[kItems][kWarps];
  uint64_t warp_sum[kWarps];
  alignas(16) uint32_t bars[kBars];
  uint32_t scan[kWarps];
  alignas(16) uint32_t cum[kBars];      // of the bars from the maximum's downwards
  float mass[kWarps];
  double table[kTable];
  uint32_t n_list;
  int found;
  uint64_t front, entry;
  uint64_t range_mass[kWarps];          // what a pass has summed of each warp's range of columns, and how many elements that were
  uint32_t range_n[kWarps];
};


template <typename T>
__global__ void __launch_bounds__(kThreads, kCtas<T>) sample_kernel(const __grid_constant__ SampleArgs p) {
  constexpr int kE = Row<T>::kE;
  extern __shared__ __align__(16) uint8_t dyn[];
  uint64_t *list = reinterpret_cast<uint64_t*>(dyn), *part = list + kCap;
  uint32_t* fine = reinterpret_cast<uint32_t*>(dyn);   // bars of all elements, where the list comes later
  __shared__ Smem<T> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank(), n_cta = cluster_size();
  const int row = blockIdx.x / n_cta;
  for (int k = tid; k < kBars; k += kThreads) sh.bars[k] = 0u;
  // (2^(a / 32) and 2^(b / 1024), of whose products the table consists: 256 x 32000 rows 64.5 us, 65.3 with an exponential for every entry)
  double* roots = reinterpret_cast<double*>(sh.cum);
  static_assert(kTable == 32 * 32 && sizeof(sh.cum) >= 64 * sizeof(double), "two times 32 roots");
  if (tid < 64) roots[tid] = exp2((double)(tid & 31) * (tid < 32 ? 1.0 / 32.0 : 1.0 / 1024.0));
  pdl_launch_dependents();
  pdl_wait();

  Row<T> r;
  r.x = static_cast<const T*>(p.x) + (int64_t)row * p.ld;
  r.maxima = reinterpret_cast<float*>(dyn + kListBytes);
  r.i0 = min(p.V, (int)rank * p.per);
  r.i1 = min(p.V, r.i0 + p.per);
  r.lead = (int)((reinterpret_cast<uintptr_t>(r.x + r.i0) & 15u) / sizeof(T));
  r.pieces = r.i1 > r.i0 ? (r.i1 - r.i0 + r.lead + kE - 1) / kE : 0;
  r.odd = false;
  r.w0 = r.lead ? 1 : 0;
  r.wn = max(0, (r.i1 - r.i0 + r.lead) / kE - r.w0);

  // ---- the row's maximum, and the histogram of the groups' maxima
  const int n_groups = (r.pieces + kThreads * kGroup - 1) / (kThreads * kGroup);
  const float temp = p.temperature[row], u = p.u[row];
  const int want_k = p.top_k ? p.top_k[row] : 0;
  const float want_p = p.top_p ? p.top_p[row] : 1.0f, min_p = p.min_p && temp < INFINITY ? p.min_p[row] : 0.0f;   // (at an infinite T all weigh 1)
  __syncthreads();   // the bars are zero
  float top = -INFINITY;
  bool odd = false;
  constexpr int kAhead = 2;   // groups whose loads are on their way
  for (int g0 = 0; g0 < n_groups; g0 += kAhead) {
    float x[kAhead][kGroup][kE];
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        const int v = ((g0 + a) * kGroup + k) * kThreads + tid;
        if (v < r.pieces) r.global(v, x[a][k]);
        else
#pragma unroll
          for (int e = 0; e < kE; ++e) x[a][k][e] = -INFINITY;
      }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      if (g0 + a >= n_groups) break;
      float most = -INFINITY;
#pragma unroll
      for (int k = 0; k < kGroup; ++k)
#pragma unroll
        for (int e = 0; e < kE; ++e) most = max_or_nan(most, x[a][k][e]);
      if (!(most <= Row<T>::kMost)) {
        odd = true;
        most = -INFINITY;
#pragma unroll
        for (int k = 0; k < kGroup; ++k)
#pragma unroll
          for (int e = 0; e < kE; ++e) most = fmaxf(most, Row<T>::clean(x[a][k][e]));
      }
      r.maxima[(g0 + a) * kThreads + tid] = most;
      top = fmaxf(top, most);
      if (most > -63.875f) atomicAdd(&sh.bars[bar_of(most)], 1u);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  int turn = 0;   // which half of `exch` is written next
  odd = __any_sync(0xffffffffu, odd);
  if (lane == 0) sh.exch[turn][warp] = order_key(top) | (odd ? 1ull << 32 : 0ull);
  cluster_arrive();
  if (temp > 0.0f)   // (while the others arrive)
    for (int j = tid; j < kTable; j += kThreads) sh.table[j] = roots[j / 32] * roots[32 + j % 32];
  cluster_wait();
  // every warp fetches what all warps of all CTAs found
  uint32_t key_max = 0u;
  for (int k = lane; k < (int)n_cta * kWarps; k += 32) {
    const uint64_t found = peer_load(&sh.exch[turn][k % kWarps], k / kWarps);
    key_max = max(key_max, (uint32_t)found);
    odd |= found >> 32 != 0ull;
  }
  key_max = __reduce_max_sync(0xffffffffu, key_max);
  r.odd = __any_sync(0xffffffffu, odd);
  turn ^= 1;
  top = key_value(key_max);

  // fn(x, column of x[0]) for the pieces from, from + step, .. below `to`, the next of which is loaded on the way (from L2); lanes without a
  // piece get -infinity.  One piece at a time: most of this code runs a few times per CTA and is itself read from L2 (256 x 150001, flat rows: 412 us,
  // 430 with two pieces on their way, 420 with two worked on at once, 427 with four)
  auto pieces_of = [&](int from, int to, int step, auto fn) MQ_INLINE {
    uint4 next = make_uint4(0u, 0u, 0u, 0u);
    if (from < to) next = r.raw(from);
#pragma unroll 1
    for (int v = from; __any_sync(0xffffffffu, v < to); v += step) {
      float x[kE];
      r.unpack(next, x);
      if (v + step < to) next = r.raw(v + step);
      if (r.odd)
#pragma unroll
        for (int e = 0; e < kE; ++e) x[e] = r.clean(x[e]);
      if (v >= to)
#pragma unroll
        for (int e = 0; e < kE; ++e) x[e] = -INFINITY;
      fn(x, r.column(v));
    }
  };

  // fn(x, column) for the elements from `least` on; groups without one are not looked at
  auto elements_from = [&](float least, auto fn) MQ_INLINE {
    for (int g = 0; g < n_groups; ++g) {
      if (!(r.maxima[g * kThreads + tid] >= least)) continue;
      float x[kGroup][kE];
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        const int v = (g * kGroup + k) * kThreads + tid;
        if (v < r.pieces) r.get(v, x[k]);
        else
#pragma unroll
          for (int e = 0; e < kE; ++e) x[k][e] = -INFINITY;
      }
      // (which they are first, then one after the other: fn once per element in line would be code that a warp reads from L2 as it goes)
      uint32_t hits = 0u;
#pragma unroll
      for (int k = 0; k < kGroup; ++k)
#pragma unroll
        for (int e = 0; e < kE; ++e) hits |= x[k][e] >= least ? 1u << (k * kE + e) : 0u;
      while (hits) {
        const int bit = __ffs((int)hits) - 1, i = r.column((g * kGroup + bit / kE) * kThreads + tid) + bit % kE;
        hits &= hits - 1u;
        fn(Row<T>::clean(r.widen(r.x[i])), i);
      }
    }
  };

  // Every thread gets the sum over all CTAs (and their warps) of each of n <= kItems numbers; sh.exch[turn ^ 1] keeps the CTA's own.  An
  // entry of `exch` is written again two sums later, when every CTA has passed the barrier behind its last reading.
  auto sum_all = [&](auto items, uint64_t* v) MQ_INLINE {
    constexpr int n = decltype(items)::value;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const uint64_t s = warp_sum(v[k]);
      if (lane == 0) sh.warp_part[k][warp] = s;
    }
    __syncthreads();
    if (tid < n) {
      uint64_t s = 0ull;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += sh.warp_part[tid][w];
      sh.exch[turn][tid] = s;
    }
    cluster_sync();
    // lane k adds up number k, from one CTA after the other
    uint64_t s = 0ull;
    if (lane < n)
      for (uint32_t q = 0; q < n_cta; ++q) s += peer_load(&sh.exch[turn][lane], q);
#pragma unroll
    for (int k = 0; k < n; ++k) v[k] = __shfl_sync(0xffffffffu, s, k);
    turn ^= 1;
  };

  if (!(top > -INFINITY)) {      // nothing to choose from
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      if (p.logp) p.logp[row] = -INFINITY;
      if (p.kept) p.kept[row] = 0;
    }
    cluster_sync();              // (a CTA stays until the others have fetched from it)
    return;
  }
  if (!(temp > 0.0f)) {          // the first of the order
    int first = INT_MAX;
    elements_from(top, [&](float, int i) { first = min(first, i); });
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0) sh.exch[turn][warp] = (uint64_t)first;
    cluster_sync();
    if (rank == 0 && warp == 0) {
      for (int k = lane; k < (int)n_cta * kWarps; k += 32) first = min(first, (int)peer_load(&sh.exch[turn][k % kWarps], k / kWarps));
      first = __reduce_min_sync(0xffffffffu, first);
      if (lane == 0) {
        p.token[row] = first;
        if (p.logp) p.logp[row] = 0.0f;
        if (p.kept) p.kept[row] = 1;
      }
    }
    cluster_sync();
    return;
  }

  __syncthreads();               // the table stands
  Weight weight;
  weight.m = (double)top;
  // exp(-40) and less rounds to 0.  Where T is below a step of x, the number below the maximum has that already: no larger factor is needed, and
  // none is taken, so that d c stays in a double's range.
  const float next = fmaxf(key_value(key_max - 1u), -FLT_MAX);
  // (rounded down: to the nearest, 40 T of 1.3 steps would be one, whose weight is not 0)
  weight.low = fmaxf(fminf(__fsub_rd(top, __fmul_ru(40.0f, temp)), next), -FLT_MAX);
  weight.c = 1.4426950408889634074 / (double)temp;
  if (next < top) weight.c = fmin(weight.c, 58.0 / ((double)top - (double)next));
  weight.table = sh.table;
  const bool low_is_0 = weight.low > -FLT_MAX;   // -infinity, lifted to it, weighs nothing either
  const bool by_k = want_k > 0 && want_k < p.V, by_p = want_p < 1.0f, by_min = min_p > 0.0f;
  // w >= min_p is x >= m - T ln(1 / min_p): the smallest float32 that is
  float x_min = -FLT_MAX;
  if (by_min) x_min = fmaxf(x_min, fminf(top, __double2float_ru((double)top + (double)temp * log((double)min_p)) + 0.0f));

  // floor(u total), and the least whole number that is not below p total
  auto share_of = [](float f, uint64_t total, bool up) -> uint64_t {
    f = f > 0.0f ? fminf(f, 0.99999994f) : 0.0f;
    const uint64_t F = (uint64_t)((double)f * 18446744073709551616.0);
    return __umul64hi(F, total) + (up && F * total != 0ull ? 1ull : 0ull);
  };
  auto mass_goal = [&](uint64_t all) { return max(1ull, (unsigned long long)share_of(want_p, all, true)); };
  auto write = [&](int token, uint64_t w, uint64_t total, int kept) {
    p.token[row] = token;
    if (p.logp) p.logp[row] = (float)log((double)w / (double)total);
    if (p.kept) p.kept[row] = kept;
  };

  // The first CTA's list: the entries of every CTA's part, n_q of them in lane q; how many they are.  Called by all behind the barrier that says
  // they are there; followed by one.
  auto fetch = [&](uint32_t n_q) MQ_INLINE -> uint32_t {
#pragma unroll
    for (int o = 1; o < kMaxCluster; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, n_q, o);
      if (lane >= o) n_q += y;
    }
    uint32_t end[kMaxCluster];
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q) end[q] = __shfl_sync(0xffffffffu, n_q, q);
    const uint32_t n = end[kMaxCluster - 1];
    if (rank == 0 && n <= (uint32_t)kCap)
      for (uint32_t k = tid; k < n; k += kThreads) {
        uint32_t q = 0, at = 0;
#pragma unroll
        for (int i = 0; i < kMaxCluster - 1; ++i)
          if (k >= end[i]) { q = i + 1; at = end[i]; }
        list[k] = peer_load(&part[k - at], q);
      }
    return n;
  };

  // ---- the elements from `least` on and below `below` that `base` keeps, as (key, index) into the first CTA's list; how many they are, or
  // -1 if too many.  Behind it no CTA needs another one's memory.
  auto gather = [&](float least, float below, const Cut& base) MQ_INLINE -> int {
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    elements_from(least, [&](float x, int i) {
      if (x < below && base.keeps(x, i)) {
        const uint32_t at = atomicAdd(&sh.n_list, 1u);
        if (at < (uint32_t)kCap) part[at] = entry_of<T>(x, i);
      }
    });
    __syncthreads();
    if (tid == 0) sh.exch[turn][0] = min(sh.n_list, (uint32_t)kCap + 1u);
    cluster_sync();
    const uint32_t mine = lane < (int)n_cta ? (uint32_t)peer_load(&sh.exch[turn][0], lane) : 0u;
    turn ^= 1;
    const uint32_t n = fetch(mine);
    cluster_sync();
    return n <= (uint32_t)kCap ? (int)n : -1;
  };

  // Of the n entries of a[] (all different), taken from the largest on: the one at which the running sum of weight_of(place) reaches `goal`
  // (1 .. the sum of all).  Eight bits at a time, from the first bit on in which they differ, by a histogram of those that have the bits
  // in front, until a bin holds one.  Called by the whole CTA.
  auto entry_at = [&](const uint64_t* a, int n, uint64_t goal, auto weight_of) MQ_INLINE -> uint64_t {
    // (The bars have been read.  A bin's sum is two words, the carry taken from what the lower one was: many entries may share a bin, and a 64-bit sum
    // in shared memory is a loop then.)
    uint32_t *low = sh.bars, *upper = low + kThreads, *number = upper + kThreads;
    static_assert(kBars >= 3 * kThreads, "three words per bin");
    uint64_t any = 0ull, both = ~0ull;
    for (int k = tid; k < n; k += kThreads)
      if (weight_of(k)) {
        any |= a[k];
        both &= a[k];
      }
    any = (uint64_t)__reduce_or_sync(0xffffffffu, (uint32_t)(any >> 32)) << 32 | __reduce_or_sync(0xffffffffu, (uint32_t)any);
    both = (uint64_t)__reduce_and_sync(0xffffffffu, (uint32_t)(both >> 32)) << 32 | __reduce_and_sync(0xffffffffu, (uint32_t)both);
    __syncthreads();
    if (lane == 0) {
      sh.warp_part[0][warp] = any;
      sh.warp_part[1][warp] = both;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      any |= sh.warp_part[0][w];
      both &= sh.warp_part[1][w];
    }
    uint64_t open = any & ~both;   // bits in which entries differ; the others need no search
    int pos = 64 - __clzll((long long)open);
    uint64_t head = pos < 64 ? any >> pos : 0ull;   // the entry's bits from pos on
    while (pos > 0) {
      const int to = max(0, pos - 8);
      __syncthreads();
      low[tid] = upper[tid] = number[tid] = 0u;
      __syncthreads();
      for (int k = tid; k < n; k += kThreads) {
        const uint64_t v = a[k], w = weight_of(k);
        if (w && (pos == 64 || v >> pos == head)) {
          const int d = (int)(v >> to) & ((1 << (pos - to)) - 1);
          const uint32_t was = atomicAdd(&low[d], (uint32_t)w), more = (uint32_t)(w >> 32) + (was + (uint32_t)w < was ? 1u : 0u);
          if (more) atomicAdd(&upper[d], more);
          atomicAdd(&number[d], 1u);
        }
      }
      __syncthreads();
      const uint64_t mine = (uint64_t)upper[255 - tid] << 32 | low[255 - tid];
      uint64_t inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (lane == 31) sh.warp_sum[warp] = inc;
      __syncthreads();
      for (int w = 0; w < warp; ++w) inc += sh.warp_sum[w];
      if (inc >= goal && inc - mine < goal) {
        sh.found = 255 - tid;
        sh.front = inc - mine;
      }
      __syncthreads();
      const int d = sh.found;
      open &= (1ull << to) - 1ull;
      const int next = 64 - __clzll((long long)open);
      head = (head << (pos - to) | (uint64_t)d) << (to - next) | (any >> next & ((1ull << (to - next)) - 1ull));
      goal -= sh.front;
      pos = next;
      if (number[d] == 1u && pos > 0) {
        for (int k = tid; k < n; k += kThreads)
          if (a[k] >> pos == head && weight_of(k)) sh.entry = a[k];
        __syncthreads();
        return sh.entry;
      }
    }
    return head;
  };
  // how many k < n satisfy `pred` (every thread calls)
  auto count_if = [&](int n, auto pred) -> int {
    int c = 0;
    for (int k0 = 0; k0 < n; k0 += kThreads) c += __syncthreads_count(k0 + tid < n && pred(k0 + tid));
    return c;
  };
  auto value_of = [](uint64_t entry) { return entry_value<T>(entry); };

  // ---- the first CTA finishes on a list that holds every kept element; S1's mass is `mass` or, with k, that of the list's first k
  auto finish_list = [&](int n, int k, uint64_t mass) MQ_INLINE {
    if (rank != 0) return;
    if (n <= kPairs) {
      // every pair compared, `share` neighbouring threads to an element
      int share = 1;
      while (share < 32 && n * share * 2 <= kThreads) share *= 2;
      const int j = tid / share, s0 = tid % share;
      const bool live = j < n;
      const uint64_t a = live ? list[j] : 0ull;
      if (tid < n) part[tid] = weight(value_of(list[tid]));
      __syncthreads();
      const uint64_t w = live ? part[j] : 0ull;
      auto sum_share = [&](uint64_t v) {
        for (int o = 1; o < share; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
      };
      auto sum_block = [&](uint64_t v) {   // of every element's own v
        v = warp_sum(s0 == 0 ? v : 0ull);
        __syncthreads();
        if (lane == 0) sh.warp_sum[warp] = v;
        __syncthreads();
        v = 0ull;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) v += sh.warp_sum[q];
        return v;
      };
      uint64_t before = 0ull;
      uint32_t place = 0u;
      for (int i = s0; i < n; i += share) {
        const bool first = list[i] > a;
        before += first ? part[i] : 0ull;
        place += first ? 1u : 0u;
      }
      before = sum_share(before);
      for (int o = 1; o < share; o <<= 1) place += __shfl_xor_sync(0xffffffffu, place, o);
      bool keep = live && (k <= 0 || place < (uint32_t)k);
      if (by_p) {
        const uint64_t all = k > 0 ? sum_block(keep ? w : 0ull) : mass;
        keep = keep && before < mass_goal(all);
      }
      if (by_min) keep = keep && (place == 0u || value_of(a) >= x_min);
      uint64_t* kept_w = list + kCap / 2;       // weights of the kept ones, 0 of the others
      if (live && s0 == 0) kept_w[j] = keep ? w : 0ull;
      const uint64_t total = sum_block(keep ? w : 0ull);
      const int kept = __syncthreads_count(keep && s0 == 0);
      uint64_t run = 0ull;                      // of those with a lower index
      for (int i = s0; i < n; i += share) run += ((uint32_t)list[i] & kIndexMask) > ((uint32_t)a & kIndexMask) ? kept_w[i] : 0ull;
      run = sum_share(run);
      const uint64_t goal = share_of(u, total, false);
      if (keep && s0 == 0 && run <= goal && goal - run < w) write(entry_index(a), w, total, kept);
      return;
    }
    // the cut, entry by entry; then the index, among those that are kept
    uint64_t cut = 0ull;             // the last entry that is kept
    auto sum_list = [&](auto weight_of) {
      uint64_t v = 0ull;
      for (int j = tid; j < n; j += kThreads) v += weight_of(j);
      v = warp_sum(v);
      __syncthreads();
      if (lane == 0) sh.warp_sum[warp] = v;
      __syncthreads();
      v = 0ull;
#pragma unroll
      for (int q = 0; q < kWarps; ++q) v += sh.warp_sum[q];
      return v;
    };
    for (int j = tid; j < n; j += kThreads) part[j] = weight(value_of(list[j]));
    __syncthreads();
    auto kept_weight = [&](int j) { return list[j] >= cut ? part[j] : 0ull; };
    if (k > 0 && k < n) cut = entry_at(list, n, (uint64_t)k, [](int) { return 1ull; });
    if (by_p) {
      const uint64_t goal = mass_goal(k > 0 ? sum_list(kept_weight) : mass);
      cut = max(cut, entry_at(list, n, goal, [&](int j) { return part[j]; }));
    }
    if (by_min) cut = max(cut, first_entry<T>(x_min));
    const uint64_t total = sum_list(kept_weight), kept = sum_list([&](int j) { return list[j] >= cut ? 1ull : 0ull; });
    // (the index in front: its order is that of the entries' lowest bits, downwards)
    uint64_t* by_index = part;
    __syncthreads();
    for (int j = tid; j < n; j += kThreads) list[j] = list[j] >= cut ? (list[j] & kIndexMask) << 32 | list[j] >> kIndexBits : 0ull;
    __syncthreads();
    const uint64_t found = entry_at(list, n, share_of(u, total, false) + 1ull, [&](int j) { return list[j] ? by_index[j] : 0ull; });
    if (tid == 0) write(entry_index(found >> 32), weight(value_of(found << kIndexBits)), total, (int)kept);
  };

  // ---- mass (or count) and count of the elements from each of the values on, of those that `base` keeps where there is one
  auto sums_from = [&](auto with_mass, auto with_base, const float (&at)[kEdges], const Cut& base, uint64_t (&mass)[kEdges], uint64_t (&count)[kEdges]) MQ_INLINE {
    constexpr bool kMass = decltype(with_mass)::value, kBase = decltype(with_base)::value;
    uint64_t m[kEdges];
    uint32_t c[kEdges];
#pragma unroll
    for (int k = 0; k < kEdges; ++k) {
      m[k] = 0ull;
      c[k] = 0u;
    }
    pieces_of(tid, r.pieces, kThreads, [&](float (&x)[kE], int column) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const uint64_t w = kMass ? weight.biased(x[e]) : 0ull;
        const bool it = !kBase || base.keeps(x[e], column + e);
#pragma unroll
        for (int k = 0; k < kEdges; ++k) {
          const bool in = it && x[e] >= at[k];
          if (kMass) m[k] += in ? w : 0ull;
          c[k] += in ? 1u : 0u;
        }
      }
    });
    uint64_t v[2 * kEdges];
#pragma unroll
    for (int k = 0; k < kEdges; ++k) {
      v[2 * k] = m[k] - (kMass ? c[k] * kBias : 0ull);
      v[2 * k + 1] = c[k];
    }
    sum_all(std::integral_constant<int, 2 * kEdges>(), v);
#pragma unroll
    for (int k = 0; k < kEdges; ++k) {
      mass[k] = v[2 * k + (kMass ? 0 : 1)];
      count[k] = v[2 * k + 1];
    }
  };

  // ---- kept elements, a warp's contiguous range at a time: weights (or ones) summed, and the first column at which the running sum exceeds
  // `at(total)`: known to the CTA that holds it, -1 elsewhere
  // (`listed` >= 0: range_mass and range_n have those above all entries of this CTA's list, which has `listed` of them)
  auto first_piece = [&](int w) { return (int)((int64_t)r.pieces * w / kWarps); };
  auto column_of = [&](auto as_weights, auto all_kept, const Cut& base, bool equal_only, const uint64_t* entries, int listed, auto at, uint64_t* total,
                       uint64_t* count) MQ_INLINE -> int {
    constexpr bool kW = decltype(as_weights)::value, kAll = decltype(all_kept)::value;
    auto term = [&](float x, int i, uint32_t* n) -> uint64_t {
      const uint64_t w = kW ? weight(x) : 1ull;
      const bool it = kAll || (base.keeps(x, i) && (!equal_only || x == base.value));
      *n += it ? 1u : 0u;
      return it ? w : 0ull;
    };
    const int a = first_piece(warp), b = first_piece(warp + 1);
    uint64_t sum = 0;
    uint32_t n = 0, terms = 0;
    if (kW && !kAll && listed >= 0) {
      for (int k = lane; k < listed; k += 32) {
        const int i = entry_index(entries[k]), piece = (i - r.i0 + r.lead) / kE;
        if (piece >= a && piece < b) sum += term(entry_value<T>(entries[k]), i, &n);
      }
      if (lane == 0) {
        sum += sh.range_mass[warp];
        n += sh.range_n[warp];
      }
    } else {
      pieces_of(a + lane, b, 32, [&](float (&x)[kE], int column) {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          if (kW && kAll) {   // (-infinity weighs nothing: all can be summed)
            sum += weight.biased(x[e]);
            n += x[e] > -INFINITY ? 1u : 0u;
          } else {
            sum += term(x[e], column + e, &n);
          }
        }
        if (kW && kAll) terms += kE;
      });
    }
    sum = warp_sum(sum - terms * kBias);
    n = __reduce_add_sync(0xffffffffu, n);
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    if (lane == 0) {
      sh.exch[turn][warp] = sum;
      atomicAdd(&sh.n_list, n);
    }
    __syncthreads();
    if (tid == 0) sh.exch[turn][kWarps] = sh.n_list;
    cluster_sync();
    // the sums of all ranges, two to a lane, and the counts
    static_assert(kMaxCluster * kWarps == 64, "two ranges to a lane");
    uint64_t s0 = 0ull, s1 = 0ull, cnt = 0ull;
    if (2 * lane < (int)n_cta * kWarps) {
      s0 = peer_load(&sh.exch[turn][(2 * lane) % kWarps], 2 * lane / kWarps);
      s1 = peer_load(&sh.exch[turn][(2 * lane + 1) % kWarps], 2 * lane / kWarps);
    }
    if (lane < (int)n_cta) cnt = peer_load(&sh.exch[turn][kWarps], lane);
    turn ^= 1;
    *count = warp_sum(cnt);
    uint64_t inc = s0 + s1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    *total = __shfl_sync(0xffffffffu, inc, 31);
    uint64_t left = at(*total);
    const uint64_t before = inc - s0 - s1;
    const bool first = left >= before && left - before < s0, second = left >= before + s0 && left < inc;
    const unsigned vote = __ballot_sync(0xffffffffu, first || second);
    int range = -1;
    if (vote) {
      const int l = __ffs(vote) - 1;
      range = 2 * l + (__shfl_sync(0xffffffffu, (int)second, l) ? 1 : 0);
      left -= __shfl_sync(0xffffffffu, second ? before + s0 : before, l);
    }
    cluster_sync();   // (the others' sums have been read)
    if (range < 0 || range / kWarps != (int)rank) return -1;
    // the range, cut among all warps; then the part it falls into, 32 pieces at a time
    const int in_warp = range % kWarps;
    const int ra = (int)((int64_t)r.pieces * in_warp / kWarps), rb = (int)((int64_t)r.pieces * (in_warp + 1) / kWarps);
    const int pa = ra + (int)((int64_t)(rb - ra) * warp / kWarps), pb = ra + (int)((int64_t)(rb - ra) * (warp + 1) / kWarps);
    sum = 0;
    pieces_of(pa + lane, pb, 32, [&](float (&x)[kE], int column) {
#pragma unroll
      for (int e = 0; e < kE; ++e) sum += term(x[e], column + e, &n);
    });
    sum = warp_sum(sum);
    if (tid == 0) sh.found = -1;
    if (lane == 0) sh.warp_sum[warp] = sum;
    __syncthreads();
    uint64_t front = 0;
    for (int w = 0; w < warp; ++w) front += sh.warp_sum[w];
    if (left >= front && left - front < sum) {
      left -= front;
      for (int v0 = pa; v0 < pb; v0 += 32) {
        const int v = v0 + lane;
        float x[kE];
        uint64_t g[kE], mine = 0;
#pragma unroll
        for (int e = 0; e < kE; ++e) g[e] = 0ull;
        if (v < pb) {
          r.get(v, x);
#pragma unroll
          for (int e = 0; e < kE; ++e) {
            g[e] = term(x[e], r.column(v) + e, &n);
            mine += g[e];
          }
        }
        uint64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint64_t y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        uint64_t run = upto - mine;
        const bool here = left >= run && left < upto;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          if (here && run <= left && left - run < g[e]) sh.found = r.column(v) + e;
          run += g[e];
        }
        if (__any_sync(0xffffffffu, here)) break;
        left -= __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    __syncthreads();
    return sh.found;
  };
  using Yes = std::integral_constant<bool, true>;
  using No = std::integral_constant<bool, false>;


  // ---- the bars of all CTAs, from the maximum's downwards: sh.cum[t] of the first t + 1.  n_bars of them, `first` is the maximum's
  int high = 0, n_bars = 0;
  float per_unit = 8.0f;
  auto edge_of = [&](int t) { return t < n_bars ? (float)(high - t) * (1.0f / per_unit) : INFINITY; };
  auto add_bars = [&](auto each, const uint32_t* bars, int first) MQ_INLINE {   // each: bars of a thread
    constexpr int kPer = decltype(each)::value;
    uint32_t n[kPer], sum = 0u;
#pragma unroll
    for (int k = 0; k < kPer; ++k) n[k] = 0u;
    if (kPer == 4) {   // (16 bytes at a time: first is one less than a multiple of four)
      for (uint32_t q = 0; q < n_cta; ++q) {
        const uint4 b = peer_load4(bars + first - 3 - 4 * tid, q);
        n[0] += b.w; n[1 % kPer] += b.z; n[2 % kPer] += b.y; n[3 % kPer] += b.x;
      }
    } else if (first >= tid) {
      for (uint32_t q = 0; q < n_cta; ++q) n[0] += peer_load(bars + first - tid, q);
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) sum += n[k];
    uint32_t inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 31) sh.scan[warp] = inc;
    __syncthreads();
    inc -= sum;
    for (int w = 0; w < warp; ++w) inc += sh.scan[w];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      inc += n[k];
      sh.cum[tid * kPer + k] = inc;
    }
    __syncthreads();
  };
  // the groups' maxima, 32 units down from the largest: as many elements as groups have a maximum there
  auto add_groups = [&]() {
    const int bar = bar_of(fmaxf(top, -64.0f));
    high = bar - kBars / 2;
    n_bars = min(kThreads, bar);   // (bar 0 takes what is far down)
    per_unit = 8.0f;
    add_bars(std::integral_constant<int, 1>(), sh.bars, bar);
  };
  // all elements, 32 units down (for top-p alone as far as there is some weight): counted along with another pass, or by one of their own.
  // Whole bars, fine_high down to fine_low: a bar counted in part would make a list of its elements longer than is known.
  const int fine_high = fine_of(fmaxf(top, -64.0f));
  const int fine_low = max(fine_high - kBars + 1, fine_of(by_k ? -64.0f : fmaxf(top - 20.0f * temp, -64.0f)));
  const float fine_from = (float)fine_low * (1.0f / 32.0f);
  int fine_state = 0;   // 1: counted, by all CTAs; 2: added up
  auto count_fine = [&](float x) {
    if (x >= fine_from) atomicAdd(&fine[fine_of(x) - fine_high + kBars - 1], 1u);
  };
  auto clear_fine = [&]() {
    __syncthreads();
    for (int k = tid; k < kBars; k += kThreads) fine[k] = 0u;
    __syncthreads();
  };
  auto add_elements = [&]() {
    if (fine_state == 0) {
      clear_fine();
      pieces_of(tid, r.pieces, kThreads, [&](float (&x)[kE], int) {
#pragma unroll
        for (int e = 0; e < kE; ++e) count_fine(x[e]);
      });
      cluster_sync();
    }
    if (fine_state < 2) {
      high = fine_high;
      n_bars = fine_high - fine_low + 1;
      per_unit = 32.0f;
      add_bars(std::integral_constant<int, kBars / kThreads>(), fine, kBars - 1);
    }
    fine_state = 2;
  };
  // the first bar at whose end there are `want`; n_bars: none
  auto bar_with = [&](uint64_t want) -> int { return count_if(n_bars, [&](int k) { return (uint64_t)sh.cum[k] < want; }); };

  // ---- top-p: the candidates, those from `edge` on that `base` keeps, with their mass; *all, the mass of S1, is added up from `own` on the way, *have
  // is theirs, *have_n how many they are.
  // kDone: they hold all that is kept, and all is done.  kTooFew: the nucleus goes on behind them.  kTooMany: it does not, but they fill more than a list.
  enum Found { kDone, kTooFew, kTooMany };
  auto candidates = [&](const Cut& base, float edge, uint64_t own, uint64_t* all, uint64_t* have, uint64_t* have_n) MQ_INLINE -> Found {
    uint64_t mass = 0ull;
    if (tid == 0) sh.n_list = 0u;
    __syncthreads();
    elements_from(edge, [&](float x, int i) {
      if (!base.keeps(x, i)) return;
      const uint32_t at = atomicAdd(&sh.n_list, 1u);
      if (at < (uint32_t)kCap) part[at] = entry_of<T>(x, i);
      mass += weight(x);
    });
    __syncthreads();
    uint64_t v[3] = {own, mass, tid == 0 ? (uint64_t)sh.n_list : 0ull};
    sum_all(std::integral_constant<int, 3>(), v);
    *all += v[0];
    *have = v[1];
    *have_n = v[2];
    if (v[1] < mass_goal(*all)) return kTooFew;
    if (v[2] > (uint64_t)kCap) return kTooMany;
    const uint32_t n = fetch(lane < (int)n_cta ? (uint32_t)peer_load(&sh.exch[turn ^ 1][2], lane) : 0u);
    cluster_sync();
    finish_list((int)n, 0, *all);
    return kDone;
  };
  // this thread's part of the mass of all that `base` keeps; the elements are counted along
  auto mass_of = [&](auto with_base, const Cut& base) MQ_INLINE -> uint64_t {
    constexpr bool kBase = decltype(with_base)::value;
    const bool counting = fine_state == 0;
    if (counting) clear_fine();
    uint64_t m = 0ull;
    uint32_t terms = 0u;
    pieces_of(tid, r.pieces, kThreads, [&](float (&x)[kE], int column) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const uint64_t w = weight.biased(x[e]);
        if (!kBase || base.keeps(x[e], column + e)) {
          m += w;
          if (kBase) ++terms;
        }
        if (counting) count_fine(x[e]);
      }
      if (!kBase) terms += kE;
    });
    return m - terms * kBias;
  };

  // ---- where the order is cut: elements are kept as long as less than `goal` (of mass or count) lies before them.  From `known_edge` on (if not
  // infinite), known_mass is known to lie, less than the goal.  *all is the mass of all, or becomes, for a
  // count and a later top-p, the mass of what is kept (0: not found on the way).  1: *base is the
  // cut.  0: all together are less.  -1: all is done, on a list.
  float few_edge = INFINITY;      // finite: the mass from it on is few_mass
  uint64_t few_mass = 0ull;
  int own_list = -1, in_ranges = -1;   // entries of this CTA's list; the same, once they and the ranges' sums say what is kept
  auto find_cut = [&](Cut* base, bool mass, uint64_t goal, uint64_t* all, float known_edge, uint64_t known_mass) MQ_INLINE -> int {
    const Cut from = *base;
    // less than the goal (above, above_n elements) lies from khi on, and no less from klo on (lo_n elements)
    uint32_t klo = order_key(-FLT_MAX), khi = key_max + 1u;
    uint64_t above = 0ull, above_n = 0ull, lo_n = ~0ull;
    add_elements();
    bool known = false;
    int listed = -1;           // entries of the list, where it holds what lies from klo on below khi
    int near, pass = -1;       // pass: the bar whose elements are listed while what lies above is summed
    uint64_t mass_above = 0ull;
    float* upto = reinterpret_cast<float*>(sh.bars);   // the guessed mass of each bar and those above it (the groups' bars have been read)
    const float kUnit = 1.0f / (float)(1ull << kPoint);
    float want = 0.0f;
    if (!mass) {
      near = bar_with(goal);   // (the counts are exact)
      known = near < n_bars;
      if (known) {
        klo = order_key(edge_of(near));
        lo_n = sh.cum[near];
        if (near > 0) {
          khi = order_key(edge_of(near - 1));
          above = above_n = sh.cum[near - 1];
        }
        if (by_p && lo_n > (uint64_t)kCap && lo_n - above_n <= (uint64_t)kCap) pass = near;
      }
    } else {
      // A bar's elements weigh about as much as its middle: that says in which bar the goal lies, as the few heavy ones, of which it would be
      // too rough, are known.  One pass sums what lies above that bar and puts its elements on a list; where the exact sums say otherwise,
      // the search below finds it.
      const int t0 = known_edge < INFINITY ? high - (int)(known_edge * 32.0f) : -1;   // (up to this bar)
      float sum = 0.0f, w4[4];
      static_assert(kBars == 4 * kThreads, "four bars to a thread");
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int t = 4 * tid + k;
        // (the numbers of a bar begin at its lower edge, and bf16's are up to its width apart: their middle is half a step lower)
        const float edge = (float)(high - t) * (1.0f / 32.0f);
        const float step = sizeof(T) == 2 ? fminf(__uint_as_float(__float_as_uint(edge) & 0x7f800000u) * (1.0f / 128.0f), 1.0f / 32.0f) : 0.0f;
        const float at = edge + 0.5f * (1.0f / 32.0f - step);
        w4[k] = t <= t0 ? 0.0f : (float)(sh.cum[t] - (t ? sh.cum[t - 1] : 0u)) * exp2f(fminf((at - top) * (float)weight.c, 0.0f));
        sum += w4[k];
      }
      float inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (lane == 31) sh.mass[warp] = inc;
      __syncthreads();
      inc -= sum;
      for (int w = 0; w < warp; ++w) inc += sh.mass[w];
      want = (float)(goal - known_mass) * kUnit;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        inc += w4[k];
        upto[4 * tid + k] = inc;
      }
      __syncthreads();
      near = count_if(kBars, [&](int t) { return upto[t] < want; });
      if (near + 1 < n_bars && sh.cum[near + 1] <= (uint32_t)kCap) {   // (a bar more, as the guess may be one too few)
        uint64_t have, have_n;
        const Found found = candidates(from, edge_of(near + 1), 0ull, all, &have, &have_n);
        if (found == kDone) return -1;
        if (found == kTooFew) {
          khi = order_key(edge_of(near + 1));
          above = have;
          above_n = have_n;
          near += 2;
        }
      }
      if (near < n_bars) pass = near;
    }
    for (int tries = 0; pass >= 0; ++tries) {
      const float e_lo = edge_of(near), e_hi = near > 0 ? edge_of(near - 1) : INFINITY;
      // (on the way, for the top-p behind: the mass of as few as its candidates are)
      const int t_few = mass ? n_bars : bar_with(kShort);
      const bool sum_few = !mass && t_few < near;
      const float e_few = sum_few ? edge_of(t_few) : INFINITY;
      uint64_t m[2] = {0ull, 0ull}, few = 0ull;
      uint32_t c = 0u, c1 = 0u;
      if (tid == 0) sh.n_list = 0u;
      __syncthreads();
      pieces_of(first_piece(warp) + lane, first_piece(warp + 1), 32, [&](float (&x)[kE], int column) {   // (a warp's range, as in column_of)
        uint32_t hits = 0u;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const uint64_t w = weight.biased(x[e]);
          if (x[e] >= e_hi) {
            m[0] += w;
            ++c;
            few += x[e] >= e_few ? w : 0ull;
          } else if (x[e] >= e_lo && from.keeps(x[e], column + e)) {
            m[1] += w;
            hits |= 1u << e;
          }
        }
        if (hits == 0u) return;
        c1 += (uint32_t)__popc(hits);
        uint32_t at = atomicAdd(&sh.n_list, (uint32_t)__popc(hits));
        for (; hits; hits &= hits - 1u, ++at) {   // (one after the other, as above)
          const int i = column + __ffs((int)hits) - 1;
          if (at < (uint32_t)kCap) part[at] = entry_of<T>(Row<T>::clean(r.widen(r.x[i])), i);
        }
      });
      __syncthreads();
      // (what `from` cuts off lies below e_hi, or the goal would not be reached there)
      uint64_t v[5] = {m[0] - c * kBias, m[1] - c1 * kBias, c, tid == 0 ? (uint64_t)sh.n_list : 0ull, few};
      if (mass) {
        const uint64_t of_warp = warp_sum(v[0]);
        const uint32_t n_warp = __reduce_add_sync(0xffffffffu, c);
        if (lane == 0) {
          sh.range_mass[warp] = of_warp;
          sh.range_n[warp] = n_warp;
        }
      }
      sum_all(std::integral_constant<int, 5>(), v);
      if (sum_few) {
        few_edge = e_few;
        few_mass = v[4] - sh.cum[t_few] * kBias;
      }
      mass_above = v[0];
      const bool exact = mass && from.value < e_hi;      // (else `from` cuts among what was summed)
      const bool low = exact && v[0] + v[1] < goal, over = exact && v[0] >= goal, right = !mass || (exact && !low && !over);
      if (over) {
        klo = order_key(e_hi);
        lo_n = v[2];
      } else if (low) {
        khi = order_key(e_lo);
        above = v[0] + v[1];
        above_n = v[2] + v[3];
      } else if (exact) {
        klo = order_key(e_lo);
        lo_n = v[2] + v[3];
        above = v[0];
        above_n = v[2];
        if (near > 0) khi = order_key(e_hi);
      }
      if ((low || over) && tries < 2) {
        // the sums say how far off the guess was there, which is most likely what it is off a few bars further, too
        want = low ? upto[near] + (float)(goal - above) * kUnit : upto[near - 1] - (float)(v[0] - goal) * kUnit;
        const int at = count_if(kBars, [&](int t) { return upto[t] < want; });
        near = low ? max(at, near + 1) : min(at, near - 1);
        if (near < n_bars) continue;
      }
      known = right;
      if (right && v[3] <= (uint64_t)kCap) {
        own_list = (int)sh.n_list;
        listed = (int)fetch(lane < (int)n_cta ? (uint32_t)peer_load(&sh.exch[turn ^ 1][3], lane) : 0u);
        cluster_sync();
      }
      break;
    }
    for (int level = 0;; ++level) {   // (from level 8 on the interval shrinks to a third of its places each time: 21 more at most)
      if (!known) {
        // Values between, downwards: some times T below the maximum and all, where nothing is known; else evenly, and in the end evenly among
        // the numbers that there are.  (Of few numbers between, some come twice.)
        float at[kEdges];
        const float lo = key_value(klo), h = fminf(key_value(khi), top);
        const bool even = level < 8 && lo > -1.0e6f && khi - klo > 64u;
#pragma unroll
        for (int k = 0; k < kEdges; ++k) {
          const float v = lo_n == ~0ull && level == 0 ? (k == 0 ? top - 8.0f * temp : -FLT_MAX) : lo + (h - lo) * ((float)(kEdges - k) / (float)(kEdges + 1));
          at[k] = level == 0 || even ? fminf(fmaxf(v, lo), h) : key_value(order_between(klo, khi, k, kEdges));
        }
        uint64_t m[kEdges], c[kEdges];
        if (!mass) sums_from(No(), No(), at, from, m, c);
        else if (from.value >= -FLT_MAX) sums_from(Yes(), Yes(), at, from, m, c);
        else sums_from(Yes(), No(), at, from, m, c);
        if (!mass && level == 0 && m[kEdges - 1] < goal) return 0;   // (of all)
        int k = 0;
#pragma unroll
        for (int e = 0; e < kEdges; ++e)
          if (k == e && m[e] < goal) {
            const uint32_t key = order_key(at[e]);
            if (key <= khi) { khi = key; above = m[e]; above_n = c[e]; }
            ++k;
          }
#pragma unroll
        for (int e = 0; e < kEdges; ++e)
          if (k == e && order_key(at[e]) >= klo) { klo = order_key(at[e]); lo_n = c[e]; }
      }
      known = false;
      if (listed < 0 && lo_n <= (uint64_t)kCap) {
        const int n = gather(key_value(klo), INFINITY, from);
        finish_list(n, mass ? 0 : (int)goal, *all);
        return -1;
      }
      if (lo_n - above_n <= (uint64_t)kCap) {
        if (listed < 0) listed = gather(key_value(klo), key_value(khi), from);
        else if (mass) in_ranges = own_list;
        // the last one before which less than the goal lies: where the running sum reaches it
        if (rank == 0) {
          for (int j = tid; j < listed; j += kThreads) part[j] = mass ? weight(value_of(list[j])) : 1ull;
          const uint64_t last = entry_at(list, listed, goal - above, [&](int j) { return part[j]; });
          uint64_t kept = 0ull;
          if (pass >= 0 && !mass)
            for (int j = tid; j < listed; j += kThreads) kept += list[j] >= last ? weight(value_of(list[j])) : 0ull;
          kept = warp_sum(kept);
          if (lane == 0) sh.warp_part[2][warp] = kept;
          __syncthreads();
          if (tid == 0) {
            for (int w = 1; w < kWarps; ++w) kept += sh.warp_part[2][w];
            sh.exch[turn][0] = last;
            sh.exch[turn][1] = mass_above + kept;
          }
        }
        cluster_sync();
        const uint64_t word = peer_load(&sh.exch[turn][0], 0);
        if (pass >= 0 && !mass) *all = peer_load(&sh.exch[turn][1], 0);
        turn ^= 1;
        *base = Cut{value_of(word), entry_index(word)};
        return 1;
      }
      if (khi - klo <= 1u || level >= kLevels) {   // thousands of equal logits: the first of them by index
        base->value = key_value(klo);
        const uint64_t g = mass ? weight(base->value) : 1ull, ties = g ? (goal - above + g - 1ull) / g : 1ull;
        uint64_t total, count;
        // (those that `from` keeps: its own cut may lie among them)
        const Cut equal{base->value, from.value == base->value ? from.idx : INT_MAX};
        const int i = column_of(No(), No(), equal, true, part, -1, [&](uint64_t t) { return min(ties, t) - 1ull; }, &total, &count);
        if (tid == 0) sh.exch[turn][0] = (uint64_t)(i + 1);
        cluster_sync();
        const uint32_t one = lane < (int)n_cta ? (uint32_t)peer_load(&sh.exch[turn][0], lane) : 0u;
        turn ^= 1;
        base->idx = (int)__reduce_max_sync(0xffffffffu, one) - 1;
        return 1;
      }
    }
  };

  Cut base{-INFINITY, INT_MIN};   // (columns in front of a slice are -inf with an index below 0)
  if (by_min && !by_k && !by_p) {
    const int n = gather(x_min, INFINITY, base);
    if (n >= 0) {
      finish_list(n, 0, 0ull);
      return;
    }
  }
  const bool short_k = by_k && want_k <= kLong;
  if (short_k || (by_p && !by_k)) add_groups();
  if (short_k) {
    const float edge = edge_of(bar_with((uint64_t)want_k));
    const int n = edge < INFINITY ? gather(edge, INFINITY, base) : -1;
    if (n >= 0) {
      finish_list(n, want_k, 0ull);
      return;
    }
  }
  uint64_t all = 0ull;
  if (by_k && find_cut(&base, false, (uint64_t)want_k, &all, INFINITY, 0ull) < 0) return;
  if (by_p) {
    float edge = few_edge;
    uint64_t have = few_mass;
    if (!(edge < INFINITY && have < mass_goal(all))) {   // (else the few are known to be too few)
      edge = edge_of(bar_with(kShort));
      uint64_t own = 0ull;
      if (all == 0ull) own = base.value >= -FLT_MAX || !low_is_0 ? mass_of(Yes(), base) : mass_of(No(), base);
      uint64_t have_n;
      if (candidates(base, edge, own, &all, &have, &have_n) == kDone) return;
      if (fine_state == 0) fine_state = 1;
    }
    const bool short_of = have < mass_goal(all);   // (else they were too many)
    if (find_cut(&base, true, mass_goal(all), &all, short_of ? edge : INFINITY, short_of ? have : 0ull) < 0) return;
  }
  if (by_min && x_min > fmaxf(base.value, -FLT_MAX)) {   // (on the cut's own value the cut's column decides)
    base = Cut{x_min, INT_MAX};
    in_ranges = -1;
  }
  uint64_t total, count;
  auto goal_of = [&](uint64_t t) { return share_of(u, t, false); };
  const int i = base.value >= -FLT_MAX || !low_is_0 ? column_of(Yes(), No(), base, false, rank == 0 ? list : part, in_ranges, goal_of, &total, &count)
                                                               : column_of(Yes(), Yes(), base, false, part, -1, goal_of, &total, &count);
  if (i >= 0 && tid == 0) write(i, weight(Row<T>::clean(r.widen(r.x[i]))), total, (int)count);
}

template <typename T>
int launch(const SampleArgs& a, int B, int cluster, int smem, cudaStream_t st) {
  // (the maxima: up to 32 groups for 2^17 columns of float32)
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, sample_kernel<T>, kListBytes + kMaximaMost)) return MQ_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)B * (unsigned)cluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, sample_kernel<T>, a);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" int mq_sample(const void* logits, int64_t ld, int32_t B, int32_t V, uint32_t flags, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const float* u, int32_t* token, float* logp, int32_t* kept, void* stream) {
  if (B < 0 || V <= 0 || (flags & ~MQ_SAMPLE_F32) || ld < V) return MQ_ERR_INVALID_ARG;
  if (V > kMaxVocab || B > (1 << 24)) return MQ_ERR_UNSUPPORTED;
  if (B == 0) return MQ_OK;
  if (!logits || !temperature || !u || !token) return MQ_ERR_INVALID_ARG;
  const int es = flags & MQ_SAMPLE_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % es) return MQ_ERR_ALIGNMENT;
  SampleArgs a{};
  a.x = logits;
  a.ld = ld;
  a.V = V;
  // as many CTAs to a row as have 2048 columns each while all of them run at once; else as have 6144 (256 rows of 32000 with filters as in
  // use: 75 us with four CTAs, 103 with eight, 83 with two; 64 rows: 41 with eight, 44 with four)
  int cluster = 1;
  while (cluster < kMaxCluster && V / (cluster * 2) >= ((int64_t)B * cluster * 2 <= sm_count() * (es == 4 ? kCtas<float> : kCtas<__nv_bfloat16>) ? 2048 : 6144)) cluster *= 2;
  a.per = ((V + cluster - 1) / cluster + 63) / 64 * 64;
  const int slice_bytes = a.per * es + 16;   // (a slice may start inside a 16-byte piece)
  const int maxima = (slice_bytes / 16 + kThreads * kGroup - 1) / (kThreads * kGroup) * kThreads * 4;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.token = token;
  a.logp = logp;
  a.kept = kept;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return es == 4 ? launch<float>(a, B, cluster, kListBytes + maxima, st) : launch<__nv_bfloat16>(a, B, cluster, kListBytes + maxima, st);
}
