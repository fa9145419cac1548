// The next token of every row of logits, from a given random number: temperature, top-k, top-p, min-p.
//
//   w_i = exp((x_i - max) / T); order: larger x first, of equal ones the lower index.  S1: the first k.  S2: those of S1 before which less
//   than p of S1's mass lies.  S3: those with w_i >= min_p.  kept = S1, S2 and S3, at least the first; the token is the first kept one in
//   index order at which the running sum of the kept weights exceeds u times their total.
//
// All three filters cut the order at one place, so the work is to find that place without sorting.
//   * A row belongs to a cluster of up to 8 CTAs; each stages its slice in shared memory (a row too long for that is read again from L2), so the
//     logits come from HBM once.  What the CTAs have to agree on (maximum, histograms, sums) goes through distributed shared memory.
//   * Weights are fixed-point numbers of 43 bits behind the point, from exponentials in double: their sums are whole numbers, the same in
//     any order, and a border between two tokens of a hundred thousand falls where 64-bit arithmetic puts it (float32 sums of such a
//     row are off by as much as a token's weight).
//   * The cut is narrowed down by histograms of 16 bins over (max - x), each thread counting (or weighing) in bins of its own, until what can
//     hold it fits into a list of 2048; mostly the whole kept set does, and one CTA finishes on the sorted list.  Large kept sets are summed
//     by warps over contiguous ranges, and only the range the random number falls into is walked.
//   * Logits that do not separate by (max - x), as thousands of equal ones, are narrowed by their bits, and ties cut by index.
#include <climits>
#include <cmath>

#include <cuda_bf16.h>

#include "mq_common.cuh"

namespace mq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBins = 16;
constexpr int kCap = 2048;            // candidates of a list
constexpr int kMaxCluster = 8;
constexpr int kItems = kBins + 1;     // what a CTA tells the others at once
constexpr int kPoint = 43;            // bits behind the point of a weight: 2^20 of them stay below 2^63
constexpr int kMaxVocab = 1 << 20;
constexpr int kTable = 64;            // 2^(j / kTable)
constexpr uint32_t kKeyNegInf = 0x007fffffu;
constexpr int kStageMax = 190 * 1024; // bytes of a staged slice

struct SampleArgs {
  const void* x;
  int64_t ld;
  int V, per;          // columns, and those of a CTA
  int staged, slice_bytes;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* token;
  float* logp;
  int32_t* kept;
};

__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

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
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void peer_store(const void* mine, uint32_t rank, uint64_t v) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(mine)), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(r), "l"(v) : "memory");
}

// an element's place: kept are keys above `key`, and of the equal ones those up to `idx`
struct Cut {
  uint32_t key;
  int idx;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= idx); }
};

// A range of the order, as the histograms narrow it down: digits of y = (max - x) c first, bits of the key then
struct Bracket {
  float c;             // y = (m - x) c
  float scale;         // 0: every y;  else floor(min(y, 15) scale) == prefix
  int prefix;
  uint32_t klo, khi;
  bool by_key;
  __device__ __forceinline__ float y_of(float m, float x) const { return x == m ? 0.0f : fminf((m - x) * c, 15.0f); }
  __device__ __forceinline__ bool holds(float y, uint32_t key) const {
    return (scale == 0.0f || (int)(y * scale) == prefix) && (!by_key || (key >= klo && key <= khi));
  }
  __device__ __forceinline__ int shift() const { return max(0, 28 - __clz((int)(khi - klo))); }
  __device__ __forceinline__ int bin(float y, uint32_t key) const {
    if (by_key) return (int)((khi - key) >> shift());
    return scale == 0.0f ? (int)y : (int)(y * scale * 16.0f) - prefix * 16;
  }
  // the part that bin d is; false: it is one key, and cannot be divided
  __device__ __forceinline__ bool narrow(int d, uint32_t key_max) {
    if (by_key) {
      const int sh = shift();
      khi -= (uint32_t)d << sh;
      if (khi - klo >= (1u << sh)) klo = khi - ((1u << sh) - 1u);
      return klo < khi;
    }
    if (scale == 0.0f) { scale = 1.0f; prefix = d; }
    else { scale *= 16.0f; prefix = prefix * 16 + d; }
    if (prefix == 15 || scale > 60000.0f) {   // the open end, or digits that float32 does not have
      by_key = true;
      klo = kKeyNegInf + 1u;
      khi = key_max;
    }
    return true;
  }
};

template <typename T>
struct Row {
  static constexpr int kE = 16 / (int)sizeof(T);   // elements of a 16-byte piece
  const T* x;          // the row
  const uint8_t* smem; // its staged slice
  int i0, i1;          // columns of this CTA
  int lead;            // elements of the first piece in front of column i0
  int pieces;
  bool staged;

  __device__ __forceinline__ float widen(T v) const;
  __device__ __forceinline__ static float clean(float v) { return v == v ? v + 0.0f : -INFINITY; }   // (NaN: never; -0 is 0)
  // columns i0 - lead + kE v ..; those that are not this CTA's read as -inf
  __device__ __forceinline__ void global(int v, float (&out)[kE]) const {
    const int first = i0 - lead + v * kE;
    if (first >= i0 && first + kE <= i1) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(x + first));
      unpack(q, out);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) out[e] = first + e >= i0 && first + e < i1 ? widen(x[first + e]) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) out[e] = clean(out[e]);
  }
  __device__ __forceinline__ void unpack(const uint4& q, float (&out)[kE]) const;
  __device__ __forceinline__ uint4 pack(const float (&in)[kE]) const;
  __device__ __forceinline__ int column(int v) const { return i0 - lead + v * kE; }
  __device__ __forceinline__ void get(int v, float (&out)[kE]) const {
    if (staged) unpack(*reinterpret_cast<const uint4*>(smem + (size_t)v * 16), out);
    else global(v, out);
  }
};
template <>
__device__ __forceinline__ float Row<float>::widen(float v) const { return v; }
template <>
__device__ __forceinline__ void Row<float>::unpack(const uint4& q, float (&out)[4]) const {
  out[0] = __uint_as_float(q.x); out[1] = __uint_as_float(q.y); out[2] = __uint_as_float(q.z); out[3] = __uint_as_float(q.w);
}
template <>
__device__ __forceinline__ uint4 Row<float>::pack(const float (&in)[4]) const {
  return make_uint4(__float_as_uint(in[0]), __float_as_uint(in[1]), __float_as_uint(in[2]), __float_as_uint(in[3]));
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
template <>
__device__ __forceinline__ uint4 Row<__nv_bfloat16>::pack(const float (&in)[8]) const {   // (values that came from bf16: exact)
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (__float_as_uint(in[2 * e]) >> 16) | (__float_as_uint(in[2 * e + 1]) & 0xffff0000u);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// exp(-(m - x) / T) as a fixed-point number.  2^t by a table of 2^(j / 64) and the exponential's series on |f| <= 1/128 (the
// first term left out is below 2^-53 of the sum); the sum with 2^(52 - kPoint) leaves the rounded number in the low bits.
struct Weight {
  double m, c;            // c = log2(e) / T
  float top;
  const double* table;
  __device__ __forceinline__ uint64_t operator()(float x) const {
    if (x == top) return 1ull << kPoint;
    const double t = (m - (double)x) * c;           // >= 0
    if (!(t < 60.0)) return 0ull;                   // (also an infinite gap times a factor of zero)
    const double magic = 6755399441055744.0 / kTable;   // 1.5 * 2^52 / kTable: adding it rounds to multiples of 1 / kTable
    const double a = magic - t;
    const double f = (magic - a) - t;               // 2^-t = 2^(-round) 2^f
    const int n = (int)(uint32_t)__double_as_longlong(a);   // -round(t * kTable), in the low bits
    const double z = f * 0.69314718055994530942;
    double p = fma(z, 1.0 / 120.0, 1.0 / 24.0);
    p = fma(p, z, 1.0 / 6.0);
    p = fma(p, z, 0.5);
    p = fma(p, z, 1.0);
    p = fma(p, z, 1.0);
    const double s = table[n & (kTable - 1)] * p;   // in (0.99, 2)
    const double w = __longlong_as_double(__double_as_longlong(s) + ((int64_t)(n >> 6) << 52));
    return (uint64_t)__double_as_longlong(w + 512.0) & ((1ull << 52) - 1ull);
  }
};
static_assert(kTable == 64 && kPoint == 43, "the shifts above");

template <typename Tx>
struct Smem {
  uint64_t exch[2][kMaxCluster][kItems];
  uint64_t warp_sum[kWarps];
  uint64_t tot[kItems];
  double table[kTable];
  uint32_t n_list, n_bin;
  int found;
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs p) {
  constexpr int kE = Row<T>::kE;
  extern __shared__ __align__(16) uint8_t dyn[];
  uint64_t* bins = reinterpret_cast<uint64_t*>(dyn);                   // [kBins][kThreads]
  uint64_t *list = bins, *part = bins + kCap;                          // (the same memory, when the bins are done with)
  static_assert(kBins * kThreads == 2 * kCap, "the lists take the bins' place");
  __shared__ Smem<T> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank(), n_cta = cluster_size();
  const int row = blockIdx.x / n_cta;
  if (tid < kTable) sh.table[tid] = exp2((double)tid / kTable);
  pdl_launch_dependents();
  pdl_wait();

  Row<T> r;
  r.x = static_cast<const T*>(p.x) + (int64_t)row * p.ld;
  r.smem = dyn + kBins * kThreads * 8;
  r.i0 = min(p.V, (int)rank * p.per);
  r.i1 = min(p.V, r.i0 + p.per);
  r.lead = (int)((reinterpret_cast<uintptr_t>(r.x + r.i0) & 15u) / sizeof(T));
  r.pieces = r.i1 > r.i0 ? (r.i1 - r.i0 + r.lead + kE - 1) / kE : 0;
  r.staged = p.staged != 0;

  int parity = 0;
  // Every CTA's n items (thread i of it holds item i) to all of them; sh.exch[parity ^ 1] afterwards
  auto exchange = [&](int n, uint64_t item) {
    if (tid < n)
      for (uint32_t q = 0; q < n_cta; ++q) peer_store(&sh.exch[parity][rank][tid], q, item);
    cluster_sync();
    parity ^= 1;
  };
  auto got = [&](uint32_t cta, int i) { return sh.exch[parity ^ 1][cta][i]; };

  // ---- the slice into shared memory, and the row's maximum
  float top = -INFINITY;
  constexpr int kU = 8;
  for (int v0 = tid; v0 < r.pieces; v0 += kThreads * kU) {
    float x[kU][kE];
#pragma unroll
    for (int k = 0; k < kU; ++k)
      if (v0 + k * kThreads < r.pieces) r.global(v0 + k * kThreads, x[k]);
#pragma unroll
    for (int k = 0; k < kU; ++k)
      if (v0 + k * kThreads < r.pieces) {
        if (r.staged) *reinterpret_cast<uint4*>(const_cast<uint8_t*>(r.smem) + (size_t)(v0 + k * kThreads) * 16) = r.pack(x[k]);
#pragma unroll
        for (int e = 0; e < kE; ++e) top = fmaxf(top, x[k][e]);
      }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) sh.warp_sum[warp] = order_key(top);
  __syncthreads();
  uint64_t best = sh.warp_sum[0];
  for (int w = 1; w < kWarps; ++w) best = max(best, sh.warp_sum[w]);
  exchange(1, best);
  for (uint32_t q = 0; q < n_cta; ++q) best = max(best, got(q, 0));
  const uint32_t key_max = (uint32_t)best;
  top = key_value(key_max);

  const float temp = p.temperature[row];
  if (key_max <= kKeyNegInf) {   // nothing to choose from
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      if (p.logp) p.logp[row] = -INFINITY;
      if (p.kept) p.kept[row] = 0;
    }
    return;
  }
  if (!(temp > 0.0f)) {          // the first of the order
    int first = INT_MAX;
    for (int v = tid; v < r.pieces; v += kThreads) {
      float x[kE];
      r.get(v, x);
#pragma unroll
      for (int e = kE - 1; e >= 0; --e)
        if (x[e] == top) first = min(first, r.column(v) + e);
    }
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0) sh.warp_sum[warp] = (uint64_t)first;
    __syncthreads();
    best = sh.warp_sum[0];
    for (int w = 1; w < kWarps; ++w) best = min(best, sh.warp_sum[w]);
    exchange(1, best);
    if (rank == 0 && tid == 0) {
      for (uint32_t q = 0; q < n_cta; ++q) best = min(best, got(q, 0));
      p.token[row] = (int32_t)best;
      if (p.logp) p.logp[row] = 0.0f;
      if (p.kept) p.kept[row] = 1;
    }
    return;
  }

  Weight weight;
  weight.m = (double)top;
  weight.top = top;
  weight.c = 1.4426950408889634074 / (double)temp;
  weight.table = sh.table;
  const int want_k = p.top_k ? p.top_k[row] : 0;
  const float want_p = p.top_p ? p.top_p[row] : 1.0f, min_p = p.min_p ? p.min_p[row] : 0.0f, u = p.u[row];
  const bool by_k = want_k > 0 && want_k < p.V, by_p = want_p < 1.0f, by_min = min_p > 0.0f;
  // w >= min_p is x >= m - T ln(1 / min_p): the smallest float32 that is
  uint32_t key_min = kKeyNegInf + 1u;
  if (by_min) {
    const float t = __double2float_ru((double)top + (double)temp * log((double)min_p));
    key_min = min(key_max, max(key_min, order_key(t + 0.0f)));
  }

  // ---- kept elements, a warp's contiguous range at a time: `value` of every one, summed; and the first column at which the
  // running sum exceeds `at(total)` (known to the CTA that holds it; *owner tells it)
  auto column_of = [&](auto value, auto at, uint64_t* total, uint64_t* count, bool* owner) -> int {
    const int a = (int)((int64_t)r.pieces * warp / kWarps), b = (int)((int64_t)r.pieces * (warp + 1) / kWarps);
    uint64_t sum = 0;
    uint32_t n = 0;
    for (int v = a + lane; v < b; v += 32) {
      float x[kE];
      r.get(v, x);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        uint64_t g;
        if (value(x[e], r.column(v) + e, &g)) { sum += g; ++n; }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    n = __reduce_add_sync(0xffffffffu, n);
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    if (lane == 0) {
      sh.warp_sum[warp] = sum;
      atomicAdd(&sh.n_list, n);
    }
    __syncthreads();
    exchange(kWarps + 1, tid < kWarps ? sh.warp_sum[tid] : (uint64_t)sh.n_list);
    uint64_t all = 0, cnt = 0;
    for (uint32_t q = 0; q < n_cta; ++q) {
      for (int w = 0; w < kWarps; ++w) all += got(q, w);
      cnt += got(q, kWarps);
    }
    *total = all;
    *count = cnt;
    uint64_t left = at(all);
    int in_warp = -1;
    *owner = false;
    for (uint32_t q = 0; q < n_cta && in_warp < 0; ++q)
      for (int w = 0; w < kWarps; ++w) {
        const uint64_t s = got(q, w);
        if (left < s) {
          in_warp = w;
          *owner = q == rank;
          break;
        }
        left -= s;
      }
    if (!*owner) return -1;
    // the range, cut among all warps; then the part it falls into, 32 pieces at a time
    const int ra = (int)((int64_t)r.pieces * in_warp / kWarps), rb = (int)((int64_t)r.pieces * (in_warp + 1) / kWarps);
    const int pa = ra + (int)((int64_t)(rb - ra) * warp / kWarps), pb = ra + (int)((int64_t)(rb - ra) * (warp + 1) / kWarps);
    sum = 0;
    for (int v = pa + lane; v < pb; v += 32) {
      float x[kE];
      r.get(v, x);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        uint64_t g;
        if (value(x[e], r.column(v) + e, &g)) sum += g;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (tid == 0) sh.found = -1;
    if (lane == 0) sh.warp_sum[warp] = sum;
    __syncthreads();
    uint64_t before = 0;
    for (int w = 0; w < warp; ++w) before += sh.warp_sum[w];
    if (left >= before && left - before < sum) {
      left -= before;
      for (int v0 = pa; v0 < pb; v0 += 32) {
        const int v = v0 + lane;
        float x[kE];
        uint64_t mine = 0;
        if (v < pb) {
          r.get(v, x);
#pragma unroll
          for (int e = 0; e < kE; ++e) {
            uint64_t g;
            if (value(x[e], r.column(v) + e, &g)) mine += g;
          }
        }
        uint64_t inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint64_t y = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += y;
        }
        const bool here = left >= inc - mine && left < inc;
        if (here) {
          uint64_t run = inc - mine;
#pragma unroll
          for (int e = 0; e < kE; ++e) {
            uint64_t g;
            if (value(x[e], r.column(v) + e, &g)) {
              if (run <= left && left < run + g) sh.found = r.column(v) + e;
              run += g;
            }
          }
        }
        if (__any_sync(0xffffffffu, here)) break;
        left -= __shfl_sync(0xffffffffu, inc, 31);
      }
    }
    __syncthreads();
    return sh.found;
  };

  // ---- a histogram of the kept elements of a bracket, over all CTAs: sh.tot
  auto histogram = [&](const Bracket& br, const Cut& base, bool mass) {
    for (int b = 0; b < kBins; ++b) bins[b * kThreads + tid] = 0ull;
    for (int v = tid; v < r.pieces; v += kThreads) {
      float x[kE];
      r.get(v, x);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const uint32_t key = order_key(x[e]);
        const float y = br.y_of(top, x[e]);
        if (base.keeps(key, r.column(v) + e) && br.holds(y, key)) bins[br.bin(y, key) * kThreads + tid] += mass ? weight(x[e]) : 1ull;
      }
    }
    __syncthreads();
    for (int b = warp; b < kBins; b += kWarps) {
      uint64_t s = 0;
      for (int k = lane; k < kThreads; k += 32) s += bins[b * kThreads + k];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) sh.tot[b] = s;
    }
    __syncthreads();
    exchange(kBins, tid < kBins ? sh.tot[tid] : 0ull);
    if (tid < kBins) {
      uint64_t s = 0;
      for (uint32_t q = 0; q < n_cta; ++q) s += got(q, tid);
      sh.tot[tid] = s;
    }
    __syncthreads();
  };

  // ---- the elements that `pick` names, as (key, index) into the first CTA's list; how many they are, or -1 if too many
  auto gather = [&](auto pick) -> int {
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    for (int v = tid; v < r.pieces; v += kThreads) {
      float x[kE];
      r.get(v, x);
#pragma unroll
      for (int e = 0; e < kE; ++e)
        if (pick(x[e], order_key(x[e]), r.column(v) + e)) {
          const uint32_t at = atomicAdd(&sh.n_list, 1u);
          if (at < (uint32_t)kCap) part[at] = (uint64_t)order_key(x[e]) << 32 | (uint32_t)~(r.column(v) + e);
        }
    }
    __syncthreads();
    const uint32_t mine = sh.n_list;
    exchange(1, mine);
    uint64_t n = 0, at = 0;
    for (uint32_t q = 0; q < n_cta; ++q) {
      if (q == rank) at = n;
      n += got(q, 0);
    }
    if (n > (uint64_t)kCap) return -1;
    for (uint32_t k = tid; k < mine; k += kThreads) peer_store(&list[at + k], 0, part[k]);
    cluster_sync();
    return (int)n;
  };

  // sorts a[0 .. n) in shared memory, largest first (a has room for the next power of two)
  auto sort_desc = [&](uint64_t* a, int n) {
    int size = 2;
    while (size < n) size <<= 1;
    for (int k = n + tid; k < size; k += kThreads) a[k] = 0ull;
    __syncthreads();
    for (int len = 2; len <= size; len <<= 1)
      for (int half = len >> 1; half > 0; half >>= 1) {
        for (int k = tid; k < size / 2; k += kThreads) {
          const int i = ((k & ~(half - 1)) << 1) | (k & (half - 1)), j = i | half;
          const uint64_t x = a[i], y = a[j];
          if ((x < y) == ((i & len) == 0)) {
            a[i] = y;
            a[j] = x;
          }
        }
        __syncthreads();
      }
  };
  // a[k] <- sum of a[0 .. k], k < n
  auto scan = [&](uint64_t* a, int n) -> uint64_t {
    const int per = (n + kThreads - 1) / kThreads, k0 = min(n, tid * per), k1 = min(n, k0 + per);
    uint64_t s = 0;
    for (int k = k0; k < k1; ++k) s += a[k];
    uint64_t inc = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 31) sh.warp_sum[warp] = inc;
    __syncthreads();
    uint64_t run = inc - s, all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) run += sh.warp_sum[w];
      all += sh.warp_sum[w];
    }
    for (int k = k0; k < k1; ++k) {
      run += a[k];
      a[k] = run;
    }
    __syncthreads();
    return all;
  };
  // how many k < n satisfy `pred` (every thread calls)
  auto count_if = [&](int n, auto pred) -> int {
    int c = 0;
    for (int k0 = 0; k0 < n; k0 += kThreads) c += __syncthreads_count(k0 + tid < n && pred(k0 + tid));
    return c;
  };

  // u and p of a total: floor(u total), and the least whole number that is not below p total
  auto share_of = [](float f, uint64_t total, bool up) -> uint64_t {
    f = f > 0.0f ? fminf(f, 0.99999994f) : 0.0f;
    const uint64_t F = (uint64_t)((double)f * 18446744073709551616.0);
    return __umul64hi(F, total) + (up && F * total != 0ull ? 1ull : 0ull);
  };
  auto write = [&](int token, uint64_t w, uint64_t total, int kept) {
    p.token[row] = token;
    if (p.logp) p.logp[row] = (float)log((double)w / (double)total);
    if (p.kept) p.kept[row] = kept;
  };

  // ---- the first CTA finishes on a list that holds every kept element; S1's mass is `mass` or, with k, that of the list's first k
  auto finish_list = [&](int n, int k, uint64_t mass) {
    if (rank != 0) return;
    sort_desc(list, n);
    if (k > 0) n = min(n, k);
    for (int j = tid; j < n; j += kThreads) part[j] = weight(key_value((uint32_t)(list[j] >> 32)));
    __syncthreads();
    int cut = n;
    if (by_p || by_min) {
      const uint64_t all = scan(part, n);
      if (by_p) {
        const uint64_t goal = max(1ull, (unsigned long long)share_of(want_p, k > 0 ? all : mass, true));
        cut = min(cut, count_if(n, [&](int j) { return (j ? part[j - 1] : 0ull) < goal; }));
      }
      if (by_min) cut = min(cut, count_if(n, [&](int j) { return (uint32_t)(list[j] >> 32) >= key_min; }));
      cut = max(cut, 1);
    }
    __syncthreads();
    // in index order: (~index, place in the list), sorted largest first
    for (int j = tid; j < cut; j += kThreads) part[j] = (list[j] & 0xffffffffull) << 32 | (list[j] >> 32);
    sort_desc(part, cut);
    for (int j = tid; j < cut; j += kThreads) list[j] = weight(key_value((uint32_t)part[j]));
    __syncthreads();
    const uint64_t total = scan(list, cut), goal = share_of(u, total, false);
    const int j = count_if(cut, [&](int i) { return list[i] <= goal; });
    if (tid == 0) write((int)~(uint32_t)(part[j] >> 32), list[j] - (j ? list[j - 1] : 0ull), total, cut);
  };

  // ---- where the order is cut: elements are kept as long as less than `goal` (count or mass; p's share of the mass, if goal is 0) lies before
  // them.  1: *base is the cut.  0: nothing is cut off.  -1: all is done, on a list.
  auto find_cut = [&](Cut* base, bool mass, uint64_t goal) -> int {
    Bracket br;
    br.c = mass ? (float)weight.c : 1.4426950408889634f;
    br.scale = 0.0f;
    br.prefix = 0;
    br.by_key = false;
    br.klo = kKeyNegInf + 1u;
    br.khi = key_max;
    uint64_t above = 0, all = 0;
    const Cut from = *base;
    for (int level = 0;; ++level) {
      histogram(br, from, mass);
      if (level == 0) {
        for (int b = 0; b < kBins; ++b) all += sh.tot[b];
        if (mass) goal = max(1ull, (unsigned long long)share_of(want_p, all, true));
        if (all < goal) return 0;
      }
      int d = 0;
      while (d < kBins - 1 && above + sh.tot[d] < goal) above += sh.tot[d++];
      const uint64_t in_bin = sh.tot[d];
      const Bracket was = br;
      const bool divisible = br.narrow(d, key_max);
      if (level == 0 && (mass || above + in_bin <= (uint64_t)kCap)) {
        // everything down to this bin
        const int n = gather([&](float x, uint32_t key, int i) { return from.keeps(key, i) && was.bin(was.y_of(top, x), key) <= d; });
        if (n >= 0) {
          finish_list(n, mass ? 0 : (int)goal, all);
          return -1;
        }
      }
      const int n = !mass && in_bin > (uint64_t)kCap ? -1
                    : gather([&](float x, uint32_t key, int i) { return from.keeps(key, i) && br.holds(br.y_of(top, x), key); });
      if (n >= 0) {
        uint64_t word = 0;
        if (rank == 0) {
          sort_desc(list, n);
          for (int j = tid; j < n; j += kThreads) part[j] = mass ? weight(key_value((uint32_t)(list[j] >> 32))) : 1ull;
          __syncthreads();
          scan(part, n);
          const int m = count_if(n, [&](int j) { return above + (j ? part[j - 1] : 0ull) < goal; });
          word = list[max(m, 1) - 1];
        }
        exchange(1, word);
        word = got(0, 0);
        base->key = (uint32_t)(word >> 32);
        base->idx = (int)~(uint32_t)word;
        return 1;
      }
      if (!divisible) {   // thousands of equal logits: the first of them by index
        const uint32_t key = br.khi;
        const uint64_t g = mass ? weight(key_value(key)) : 1ull, ties = g ? (goal - above + g - 1) / g : 1ull;
        uint64_t total, count;
        bool owner;
        const int i = column_of([&](float x, int c, uint64_t* one) { *one = 1ull; return order_key(x) == key && from.keeps(key, c); },
                                [&](uint64_t t) { return min(ties, t) - 1; }, &total, &count, &owner);
        exchange(1, owner ? (uint64_t)(i + 1) : 0ull);
        uint64_t at = 0;
        for (uint32_t q = 0; q < n_cta; ++q) at |= got(q, 0);
        base->key = key;
        base->idx = (int)at - 1;
        return 1;
      }
    }
  };

  Cut base{kKeyNegInf, INT_MIN};   // (columns in front of a slice are -inf with an index below 0)
  if (by_k && find_cut(&base, false, (uint64_t)want_k) < 0) return;
  if (by_p && find_cut(&base, true, 0ull) < 0) return;
  if (by_min && key_min > base.key) base = Cut{key_min - 1u, INT_MIN};
  if (by_min && !by_k && !by_p) {
    const int n = gather([&](float, uint32_t key, int i) { return base.keeps(key, i); });
    if (n >= 0) {
      finish_list(n, 0, 0ull);
      return;
    }
  }
  uint64_t total, count;
  bool owner;
  const int i = column_of([&](float x, int c, uint64_t* g) {
                            if (!base.keeps(order_key(x), c)) return false;
                            *g = weight(x);
                            return true;
                          },
                          [&](uint64_t t) { return share_of(u, t, false); }, &total, &count, &owner);
  if (owner && tid == 0 && i >= 0) write(i, weight(Row<T>::clean(r.widen(r.x[i]))), total, (int)count);
}

template <typename T>
int launch(const SampleArgs& a, int B, int cluster, cudaStream_t st) {
  const int smem = kBins * kThreads * 8 + (a.staged ? a.slice_bytes : 0);
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, sample_kernel<T>, kBins * kThreads * 8 + kStageMax)) return MQ_ERR_CUDA;
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
  // as many CTAs to a row as have 2048 columns each
  int cluster = 1;
  while (cluster < kMaxCluster && V / (cluster * 2) >= 2048) cluster *= 2;
  a.per = ((V + cluster - 1) / cluster + 63) / 64 * 64;
  a.slice_bytes = a.per * es + 16;   // (the slice may start inside a 16-byte piece)
  a.slice_bytes = (a.slice_bytes + 15) / 16 * 16;
  a.staged = a.slice_bytes <= kStageMax;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.token = token;
  a.logp = logp;
  a.kept = kept;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return es == 4 ? launch<float>(a, B, cluster, st) : launch<__nv_bfloat16>(a, B, cluster, st);
}
