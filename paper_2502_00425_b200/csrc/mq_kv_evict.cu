// Eviction from the paged cache by accumulated weight: per sequence and key/value head the first n_first and the last
// n_last keys stay, and of the others those with the largest weight (equal ones: the lowest index first) until the
// budget is full; the kept rows move, in their order, to fresh pages.
//
// Two kernels.  Selection: one CTA per (sequence, head) finds the weight of the last kept key exactly by a radix select
// over the weights' order-preserving integer images (12, 10 and 10 bits), then writes the kept indices in order with
// block-wide prefix counts.  The images of up to kHeld keys stay in shared memory (the weights are read once, and two CTAs
// fit an SM); longer sequences are read again for each pass.  Copy: 16-byte pieces of all kept
// rows of the batch, many in flight per thread; this is what the call's bytes are.  32 sequences of 700 to 16384 keys, 8 heads of
// 128 in bf16, cut to 2000: 104 us for 463 MB (4.4 TB/s): 78 of copying rows of 256 bytes from anywhere (5.4 TB/s), 20 of selection.
#include "mq_kv.cuh"

namespace mq {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kBins = 4096;

struct EvictParams {
  KvView src, dst;
  int dim_bytes;
  const int32_t* table;
  int max_pages;
  const int32_t* kv_len;
  int n_seq;
  const float* W;
  int64_t w_seq, w_head;
  int w_keys;   // entries of a row of W; keys behind it count as NaN
  int budget, n_first, n_last;
  const int32_t* dst_table;
  int dst_max_pages;
  int32_t* kept;
  int32_t* new_len;
  float* W_out;
};

__device__ __forceinline__ int evict_len(const EvictParams& p, int b) {
  return (int)min((int64_t)max(__ldcg(p.kv_len + b), 0), (int64_t)p.max_pages << p.src.page_shift);
}

// Larger weights have larger images; NaN has the smallest, and the two zeros are one.
__device__ __forceinline__ uint32_t image(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Block-wide exclusive prefix of two 16-bit counts packed in one word (a thread counts at most 4: 4096 in all).
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t* red, uint32_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) red[warp] = inc;
  __syncthreads();
  const uint32_t w = lane < kSelWarps ? red[lane] : 0u;
  uint32_t winc = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, winc, o);
    if (lane >= o) winc += y;
  }
  total = __shfl_sync(0xffffffffu, winc, 31);
  const uint32_t base = __shfl_sync(0xffffffffu, winc - w, warp);
  __syncthreads();   // `red` may be written again
  return base + inc - v;
}

constexpr int kHeld = 24576;   // images kept in shared memory: 96 KB, two CTAs to an SM

__global__ void __launch_bounds__(kSelThreads, 2)
kv_select_kernel(const __grid_constant__ EvictParams p, const int held_most) {
  extern __shared__ __align__(16) uint32_t img[];   // [held_most rounded up to 4]
  __shared__ __align__(16) uint32_t hist[kBins];
  __shared__ uint32_t red[32];
  __shared__ uint32_t found[2];
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  reinterpret_cast<uint4*>(hist)[tid] = make_uint4(0u, 0u, 0u, 0u);
  pdl_wait();
  pdl_launch_dependents();   // (behind the wait: the copy kernel reads lengths and tables before its own)
  const int n = evict_len(p, b);
  const float* row = p.W + (int64_t)b * p.w_seq + (int64_t)g * p.w_head;
  const int n_w = min(n, p.w_keys);
  auto w = [&](int j) { return j < n_w ? row[j] : __int_as_float(0x7fffffff); };
  const int64_t out = ((int64_t)b * p.src.n_kv_heads + g) * p.budget;
  // (kv_len and new_len may be one array: it is written once every head has been selected, by the copy)
  if (p.budget == 0 && g == 0 && tid == 0) p.new_len[b] = 0;
  if (n <= p.budget) {
    for (int j = tid; j < n; j += kSelThreads) {
      p.kept[out + j] = j;
      if (p.W_out) p.W_out[out + j] = w(j);
    }
    return;
  }
  const int lo = p.n_first, hi = n - p.n_last;     // the keys that compete
  uint32_t need = (uint32_t)(p.budget - p.n_first - p.n_last);   // how many of them stay; < hi - lo
  const bool held = n <= held_most;
  uint32_t prefix = 0u, known = 0u;                // the bits of the last kept image found so far
  __syncthreads();                                 // the bins are zero
  // the first pass counts while it reads the weights
  for (int j0 = tid; j0 < n; j0 += 4 * kSelThreads) {
    float v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = w(j0 + c * kSelThreads);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int j = j0 + c * kSelThreads;
      if (j >= n) break;
      const uint32_t u = image(v[c]);
      if (held) img[j] = u;
      if (j >= lo && j < hi) atomicAdd(&hist[u >> 20], 1u);
    }
  }
  __syncthreads();
  if (need > 0) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 20 : pass == 1 ? 10 : 0;
      const uint32_t bins = pass == 0 ? 4096u : 1024u;
      if (pass > 0) {
        for (int j = lo + tid; j < hi; j += kSelThreads) {
          const uint32_t u = held ? img[j] : image(w(j));
          if ((u & known) == prefix) atomicAdd(&hist[(u >> shift) & 1023u], 1u);
        }
        __syncthreads();
      }
      // from the largest bin down: the bin in which the count reaches `need`.  A thread has 4 bins, or 1.
      uint32_t h[4] = {0u, 0u, 0u, 0u};
      const uint32_t bin0 = pass == 0 ? 4095u - 4u * (uint32_t)tid : 1023u - (uint32_t)tid;   // its largest bin
      if (pass == 0) {
        const uint4 x = reinterpret_cast<const uint4*>(hist)[kSelThreads - 1 - tid];
        h[0] = x.w; h[1] = x.z; h[2] = x.y; h[3] = x.x;
      } else {
        h[0] = hist[bin0];
      }
      const uint32_t mine = h[0] + h[1] + h[2] + h[3];
      uint32_t inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (lane == 31) red[warp] = inc;
      __syncthreads();
      const uint32_t sum = red[lane];            // warp sums, scanned by every warp
      uint32_t before = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += y;
      }
      before = __shfl_sync(0xffffffffu, before - sum, warp) + inc - mine;
      if (before < need && before + mine >= need) {
        uint32_t acc = before;
#pragma unroll
        for (uint32_t c = 0; c < 4u; ++c) {
          if (acc < need && acc + h[c] >= need) {
            found[0] = bin0 - c;
            found[1] = need - acc;
          }
          acc += h[c];
        }
      }
      if (pass < 2) hist[tid] = 0u;              // (every thread has read its bins; the next pass has 1024 of them)
      __syncthreads();
      prefix |= found[0] << shift;
      known |= (bins - 1u) << shift;
      need = found[1];
    }
  }
  // every competing key with an image above `prefix` stays, and the first `need` of those equal to it (need = 0: none do)
  const bool any = known != 0u;
  uint32_t above = 0u, equal = 0u;   // counts before these keys
  for (int j0 = tid * 4; j0 - tid * 4 < n; j0 += 4 * kSelThreads) {
    uint32_t u[4] = {0u, 0u, 0u, 0u};
    if (held) {
      if (j0 < n) {
        const uint4 x = *reinterpret_cast<const uint4*>(img + j0);
        u[0] = x.x; u[1] = x.y; u[2] = x.z; u[3] = x.w;
      }
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (j0 + c < n) u[c] = image(w(j0 + c));
    }
    uint32_t cls = 0u, cnt = 0u;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int j = j0 + c;
      if (j >= n) continue;
      if (j < lo || j >= hi || (any && u[c] > prefix)) { cls |= 1u << (2 * c); cnt += 1u; }
      else if (any && u[c] == prefix) { cls |= 2u << (2 * c); cnt += 1u << 16; }
    }
    uint32_t total;
    const uint32_t pre = block_prefix(cnt, red, total);
    uint32_t a = above + (pre & 0xffffu), e = equal + (pre >> 16);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t k = (cls >> (2 * c)) & 3u;
      if (k == 1u || (k == 2u && e < need)) {
        const int64_t at = out + a + min(e, need);
        p.kept[at] = j0 + c;
        if (p.W_out) p.W_out[at] = w(j0 + c);
      }
      if (k == 1u) ++a;
      if (k == 2u) ++e;
    }
    above += total & 0xffffu;
    equal += total >> 16;
  }
}

// Threads walk the 16-byte pieces of all kept rows: piece q of row i of head g of sequence b.
constexpr int kCopyThreads = 256;
constexpr int kCopyRows = 4;   // rows a lane has in flight

template <int kRowBytes>
__global__ void __launch_bounds__(kCopyThreads)
kv_copy_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kPieces = kRowBytes / 16, kPerCta = kCopyThreads / kPieces;   // rows per CTA and step
  // What came before the selection is complete once this kernel runs (every CTA of the selection has passed its own wait before
  // it lets this one start); only the kept indices have to be waited for.
  const int b = blockIdx.z, g = blockIdx.y;
  const int m = min(evict_len(p, b), p.budget);
  const int pc = (int)threadIdx.x % kPieces, r = (int)threadIdx.x / kPieces;
  const int32_t* kept = p.kept + ((int64_t)b * p.src.n_kv_heads + g) * p.budget;
  pdl_launch_dependents();
  pdl_wait();
  if (blockIdx.x == 0 && g == 0 && threadIdx.x == 0) p.new_len[b] = m;   // (CTAs that read it from here get the same m)
  for (int i0 = blockIdx.x * kPerCta * kCopyRows; i0 < m; i0 += gridDim.x * kPerCta * kCopyRows) {
    uint4 k[kCopyRows], v[kCopyRows];
    int64_t to[kCopyRows];
#pragma unroll
    for (int c = 0; c < kCopyRows; ++c) {
      const int i = i0 + c * kPerCta + r;
      k[c] = v[c] = make_uint4(0u, 0u, 0u, 0u);
      to[c] = -1;
      if (i >= m) continue;
      const int j = kept[i];
      const int from_page = p.table[(int64_t)b * p.max_pages + (j >> p.src.page_shift)];
      const int to_page = p.dst_table[(int64_t)b * p.dst_max_pages + (i >> p.dst.page_shift)];
      if ((unsigned)from_page < (unsigned)p.src.n_pages) {
        const int64_t off = (int64_t)from_page * p.src.page_stride + (int64_t)g * p.src.head_stride +
                            (int64_t)(j & ((1 << p.src.page_shift) - 1)) * p.src.slot_stride + pc * 16;
        k[c] = *reinterpret_cast<const uint4*>(p.src.K + off);
        v[c] = *reinterpret_cast<const uint4*>(p.src.V + off);
      }
      if ((unsigned)to_page < (unsigned)p.dst.n_pages)
        to[c] = (int64_t)to_page * p.dst.page_stride + (int64_t)g * p.dst.head_stride +
                (int64_t)(i & ((1 << p.dst.page_shift) - 1)) * p.dst.slot_stride + pc * 16;
    }
#pragma unroll
    for (int c = 0; c < kCopyRows; ++c) {
      if (to[c] < 0) continue;
      *reinterpret_cast<uint4*>(const_cast<uint8_t*>(p.dst.K) + to[c]) = k[c];
      *reinterpret_cast<uint4*>(const_cast<uint8_t*>(p.dst.V) + to[c]) = v[c];
    }
  }
}

template <int kRowBytes>
cudaError_t launch_copy(const EvictParams& p, cudaStream_t st) {
  constexpr int rows = kCopyThreads / (kRowBytes / 16) * kCopyRows;
  const unsigned x = (unsigned)((p.budget + rows - 1) / rows);
  return launch_pdl(kv_copy_kernel<kRowBytes>, dim3(x < 1024u ? x : 1024u, (unsigned)p.src.n_kv_heads, (unsigned)p.n_seq),
                    dim3(kCopyThreads), 0, st, p);
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" int mq_kv_evict(const mq_kv_cache* cache, const int32_t* page_table, int32_t max_pages, const int32_t* kv_len,
                           int32_t n_seq, const float* W, int64_t w_seq_stride, int64_t w_head_stride, int32_t w_keys, int32_t budget,
                           int32_t n_first, int32_t n_last, const mq_kv_cache* dst, const int32_t* dst_table,
                           int32_t dst_max_pages, int32_t* kept, int32_t* new_len, float* W_out, void* stream) {
  EvictParams p{};
  int rc = check_kv_cache(cache, &p.src);
  if (rc != MQ_OK) return rc;
  if ((rc = check_kv_cache(dst, &p.dst)) != MQ_OK) return rc;
  if (dst->flags != cache->flags || dst->head_dim != cache->head_dim || dst->n_kv_heads != cache->n_kv_heads || !kv_rows_apart(dst)) return MQ_ERR_INVALID_ARG;
  if (n_seq < 0 || max_pages < 0 || dst_max_pages < 0 || budget < 0 || n_first < 0 || n_last < 0 || w_seq_stride < 0 || w_head_stride < 0 || w_keys < 0)
    return MQ_ERR_INVALID_ARG;
  if ((int64_t)n_first + n_last > budget || (int64_t)dst_max_pages * dst->page_size < budget) return MQ_ERR_INVALID_ARG;
  if (n_seq > kMaxKvSeqs || cache->n_kv_heads > 65535 || max_pages > (1 << 22) || dst_max_pages > (1 << 22)) return MQ_ERR_UNSUPPORTED;
  if (n_seq == 0) return MQ_OK;
  if (!kv_len || !new_len || (max_pages > 0 && (!page_table || (w_keys > 0 && !W))) || (budget > 0 && (!dst_table || !kept))) return MQ_ERR_INVALID_ARG;
  // lengths in place are fine, as one array; shifted ones would be read after they were written
  if (kv_len != new_len && kv_len < new_len + n_seq && new_len < kv_len + n_seq) return MQ_ERR_INVALID_ARG;
  // a head's kept weights would replace weights that other heads still have to read
  if (W_out && W && budget > 0 && w_keys > 0) {
    const __int128 w_end = (__int128)(n_seq - 1) * w_seq_stride + (__int128)(cache->n_kv_heads - 1) * w_head_stride + w_keys;
    const __int128 out_end = (__int128)n_seq * cache->n_kv_heads * budget, w0 = reinterpret_cast<intptr_t>(W), o0 = reinterpret_cast<intptr_t>(W_out);
    if (w0 < o0 + out_end * 4 && o0 < w0 + w_end * 4) return MQ_ERR_INVALID_ARG;
  }
  p.dim_bytes = cache->head_dim * ((cache->flags & MQ_KV_INT8) ? 1 : 2);
  p.table = page_table; p.max_pages = max_pages; p.kv_len = kv_len; p.n_seq = n_seq;
  p.W = W; p.w_seq = w_seq_stride; p.w_head = w_head_stride; p.w_keys = w_keys;
  p.budget = budget; p.n_first = n_first; p.n_last = n_last;
  p.dst_table = dst_table; p.dst_max_pages = dst_max_pages;
  p.kept = kept; p.new_len = new_len; p.W_out = W_out;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_select_kernel, kHeld * 4)) return MQ_ERR_CUDA;
  const int64_t reach = (int64_t)max_pages * cache->page_size;
  const int held = reach <= budget ? 0 : reach < kHeld ? (int)reach : kHeld;
  cudaError_t e = launch_pdl(kv_select_kernel, dim3((unsigned)cache->n_kv_heads, (unsigned)n_seq), dim3(kSelThreads), (size_t)align_up(held, 4) * 4, st,
                             p, held);
  if (e == cudaSuccess && budget > 0)
    e = p.dim_bytes == 256 ? launch_copy<256>(p, st) : p.dim_bytes == 128 ? launch_copy<128>(p, st) : launch_copy<64>(p, st);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}
