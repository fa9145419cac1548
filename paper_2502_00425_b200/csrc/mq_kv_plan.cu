// A step's bookkeeping on the GPU: which pages the sequences of a paged cache get or give back, and where the step's rows go.
//
//   A sequence of l keys keeps k = min(keep, l) and grows by n: with p(x) = ceil(x / page_size), the entries p(k + n) .. p(l) - 1 of its
//   table row go back to the free list, or p(l) .. p(k + n) - 1 are taken from it.  (Cut down inside its borrowed pages, it gives back
//   all of its own and takes what it needs anew.)  Pages go back first: with top = n_free + all that go back, the i-th of them, in the
//   order of sequence and entry, becomes free[top - 1 - i], and the i-th that is taken is free[top - 1 - i].  A step that takes another
//   one back so leaves the list as it was.
//   Row j of sequence b goes to slot table[b][(k + j) / page_size] * page_size + (k + j) % page_size.
//
// The first kernel is one block: a prefix over at most 2048 sequences (rows, pages back, pages taken), all checks before anything is
// written, then a thread per page that moves.  The second has a thread per row, which finds its sequence by bisection; up to
// kOneLaunch rows the first kernel does that too.  Both are bound by latency: the launch, the lengths' loads, the scan, the chain free list ->
// table -> slot.  A step of 256 sequences and the one that takes it back: 12.1 us captured, 64 prompts with 57000 rows 15.5.
#include <climits>

#include "mq_kv.cuh"

namespace mq {
namespace {

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;   // (256 for up to 256 sequences: no faster, and slower where many pages move)
constexpr int kRowThreads = 256;
constexpr int kOneLaunch = 4096;

struct PlanArgs {
  int n_seq, max_pages, page_shift, n_pages;
  int32_t *kv_len, *seen, *table, *borrowed, *free_pages, *n_free;
  const int32_t *new_len, *keep;
  int max_rows;
  int32_t* cu_q;
  int64_t* slots;
  int32_t *pos, *status;
};

// the last b < n with at[b] <= i; at is non-decreasing from 0 and i < at[n]
__device__ __forceinline__ int bisect(const int32_t* at, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Row r of the step; the lengths, positions and tables are the new ones
__device__ __forceinline__ void place_row(const PlanArgs& p, const int32_t* cu, const int32_t* len, const int32_t* seen, int r) {
  if (r >= cu[p.n_seq]) {
    p.slots[r] = -1;
    p.pos[r] = 0;
    return;
  }
  const int b = bisect(cu, p.n_seq, r), to_end = cu[b + 1] - r;
  const int j = len[b] - to_end, page = p.table[(int64_t)b * p.max_pages + (j >> p.page_shift)];
  p.slots[r] = page < 0 ? -1 : ((int64_t)page << p.page_shift) + (j & ((1 << p.page_shift) - 1));
  p.pos[r] = seen[b] - to_end;
}

// kPer: sequences of a thread
template <int kPer>
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(const __grid_constant__ PlanArgs p, const bool place) {
  constexpr int kThreads = kPlanThreads, kWarps = kPlanWarps, kSeqs = kPer * kThreads;
  __shared__ int32_t cu[kSeqs + 1], back_at[kSeqs + 1], take_at[kSeqs + 1];
  __shared__ int32_t back_from[kSeqs], take_from[kSeqs];   // first table entry that goes back, that is taken
  __shared__ int64_t red[3][kWarps];
  __shared__ int site;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = p.n_seq;
  if (tid == 0) site = INT_MAX;
  pdl_launch_dependents();
  pdl_wait();
  __syncthreads();
  const int page = 1 << p.page_shift, mask = page - 1;
  const int64_t reach = (int64_t)p.max_pages << p.page_shift;
  const int n_free = *p.n_free;
  int64_t sum[3] = {0, 0, 0};      // rows, pages back, pages taken
  int count[kPer][3], len[kPer], seen[kPer], lent[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = tid * kPer + k;
    count[k][0] = count[k][1] = count[k][2] = len[k] = seen[k] = lent[k] = 0;
    if (b >= n) continue;
    const int old = p.kv_len[b], want = p.new_len[b], lim = p.keep ? p.keep[b] : old, had = p.borrowed ? p.borrowed[b] : 0, was = p.seen[b];
    if (old < 0 || old > reach || want < 0 || lim < 0 || had < 0 || (int64_t)had << p.page_shift > old) {
      atomicMin(&site, 1);
      continue;
    }
    const int kept = min(lim, old);
    const int64_t to = (int64_t)kept + want;
    const bool inside = kept < (int64_t)had << p.page_shift;   // of the borrowed pages, which are not written to
    if (to > reach || (inside && (kept & mask))) {
      atomicMin(&site, 1);
      continue;
    }
    const int p0 = (int)(((int64_t)old + mask) >> p.page_shift), p2 = (int)((to + mask) >> p.page_shift);
    lent[k] = inside ? kept >> p.page_shift : had;
    const int from = inside ? had : min(p0, p2), first = inside ? lent[k] : p0;
    count[k][0] = want;
    count[k][1] = p0 - from;
    count[k][2] = max(0, p2 - first);
    len[k] = (int)to;
    seen[k] = (kept > 0 ? was - (old - kept) : 0) + want;
    back_from[b] = from;
    take_from[b] = first;
#pragma unroll
    for (int c = 0; c < 3; ++c) sum[c] += count[k][c];
  }
  // prefixes over the sequences
  int64_t at[3], all[3] = {0, 0, 0};
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    int64_t inc = sum[c];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31) red[c][warp] = inc;
    at[c] = inc - sum[c];
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < 3; ++c) {   // (every warp over the sums of all: lane w has that of warp w)
    const int64_t own = lane < kWarps ? red[c][lane] : 0;
    int64_t inc = own;
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    at[c] += __shfl_sync(0xffffffffu, inc - own, warp);
    all[c] = __shfl_sync(0xffffffffu, inc, kWarps - 1);
  }
  const int64_t top = (int64_t)n_free + all[1];
  int why = site;
  if (why == INT_MAX) why = all[0] > p.max_rows ? 2 : n_free < 0 || top > p.n_pages ? 3 : all[2] > top ? 4 : 0;
  if (why) {   // nothing is changed, and the step has no rows
    for (int b = tid; b <= n; b += kThreads) p.cu_q[b] = 0;
    if (place)
      for (int r = tid; r < p.max_rows; r += kThreads) { p.slots[r] = -1; p.pos[r] = 0; }
    if (tid == 0 && p.status && atomicCAS(p.status, MQ_OK, why == 4 ? MQ_ERR_WORKSPACE : MQ_ERR_INVALID_ARG) == MQ_OK) p.status[1] = why;
    return;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int b = tid * kPer + k;
    if (b >= n) break;
    cu[b] = (int)at[0];
    back_at[b] = (int)at[1];
    take_at[b] = (int)at[2];
    p.cu_q[b] = (int)at[0];
    p.kv_len[b] = len[k];
    p.seen[b] = seen[k];
    if (p.borrowed) p.borrowed[b] = lent[k];
#pragma unroll
    for (int c = 0; c < 3; ++c) at[c] += count[k][c];
  }
  if (tid == 0) {
    cu[n] = (int)all[0];
    back_at[n] = (int)all[1];
    take_at[n] = (int)all[2];
    p.cu_q[n] = (int)all[0];
    *p.n_free = (int)(top - all[2]);
  }
  __syncthreads();
  for (int i = tid; i < (int)all[1]; i += kThreads) {
    const int b = bisect(back_at, n, i);
    p.free_pages[top - 1 - i] = p.table[(int64_t)b * p.max_pages + back_from[b] + (i - back_at[b])];
  }
  __syncthreads();
  for (int i = tid; i < (int)all[2]; i += kThreads) {
    const int b = bisect(take_at, n, i);
    p.table[(int64_t)b * p.max_pages + take_from[b] + (i - take_at[b])] = p.free_pages[top - 1 - i];
  }
  if (!place) return;
  __syncthreads();
  int32_t *len_s = back_from, *seen_s = take_from;   // (whose entries have moved)
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (tid * kPer + k < n) {
      len_s[tid * kPer + k] = len[k];
      seen_s[tid * kPer + k] = seen[k];
    }
  __syncthreads();
  for (int r = tid; r < p.max_rows; r += kThreads) place_row(p, cu, len_s, seen_s, r);
}

__global__ void __launch_bounds__(kRowThreads) kv_plan_rows_kernel(const __grid_constant__ PlanArgs p) {
  __shared__ int32_t cu[kMaxKvSeqs + 1];
  pdl_launch_dependents();
  pdl_wait();
  for (int b = threadIdx.x; b <= p.n_seq; b += kRowThreads) cu[b] = p.cu_q[b];
  __syncthreads();
  const int r = blockIdx.x * kRowThreads + threadIdx.x;
  if (r < p.max_rows) place_row(p, cu, p.kv_len, p.seen, r);
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" int mq_kv_plan(const mq_kv_state* s, const int32_t* new_len, const int32_t* keep, int32_t max_rows, int32_t* cu_q, int64_t* slots,
                          int32_t* pos, int32_t* status, void* stream) {
  if (!s || s->n_seq < 0 || s->max_pages < 0 || s->n_pages < 0 || max_rows < 0 || s->page_size <= 0) return MQ_ERR_INVALID_ARG;
  if (s->n_seq > kMaxKvSeqs || s->max_pages > (1 << 22) || max_rows > (1 << 30)) return MQ_ERR_UNSUPPORTED;
  if (s->page_size < 16 || s->page_size > 256 || (s->page_size & (s->page_size - 1))) return MQ_ERR_UNSUPPORTED;
  if (!cu_q || !s->n_free) return MQ_ERR_INVALID_ARG;
  if (s->n_seq > 0 && (!s->kv_len || !s->seen || !new_len || (s->max_pages > 0 && !s->page_table))) return MQ_ERR_INVALID_ARG;
  if ((s->n_pages > 0 && !s->free_pages) || (max_rows > 0 && (!slots || !pos))) return MQ_ERR_INVALID_ARG;
  PlanArgs p{};
  p.n_seq = s->n_seq;
  p.max_pages = s->max_pages;
  p.page_shift = 31 - __builtin_clz((unsigned)s->page_size);
  p.n_pages = s->n_pages;
  p.kv_len = s->kv_len;
  p.seen = s->seen;
  p.table = s->page_table;
  p.borrowed = s->borrowed;
  p.free_pages = s->free_pages;
  p.n_free = s->n_free;
  p.new_len = new_len;
  p.keep = keep;
  p.max_rows = max_rows;
  p.cu_q = cu_q;
  p.slots = slots;
  p.pos = pos;
  p.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool place = max_rows <= kOneLaunch;
  cudaError_t e = s->n_seq <= kPlanThreads ? launch_pdl(kv_plan_kernel<1>, dim3(1), dim3(kPlanThreads), 0, st, p, place)
                                           : launch_pdl(kv_plan_kernel<kMaxKvSeqs / kPlanThreads>, dim3(1), dim3(kPlanThreads), 0, st, p, place);
  if (e == cudaSuccess && !place)
    e = launch_pdl(kv_plan_rows_kernel, dim3((unsigned)((max_rows + kRowThreads - 1) / kRowThreads)), dim3(kRowThreads), 0, st, p);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}
