// How the attention kernels over a paged cache divide their work (mq_kv_attn.cu, mq_kv_chunk.cu).
//
// A UNIT is (sequence, key/value head, block of query rows); a query row is (token, query head of the group), token
// major, so that the heads of a group share every key tile.  A unit walks its keys in tiles.  All units form one line, a
// unit as long as its tiles plus a fixed length for what it costs besides them (queries, filling the pipeline, writing
// the result), and the line is cut into equal contiguous ranges, one per worker (CTA): ragged batches, one long
// sequence and many short ones are all balanced without the host knowing a length.  A worker whose range covers a
// unit's tiles whole writes its output; otherwise it leaves a partial result (exponent reference, sum, unnormalised
// output) in its slot and the combine kernel joins the slots in the order of the keys: no atomics, the result does
// not depend on timing.
//
// Sequences that share a prefix (mq_kv_attention_shared) go over two lines, each with the same kernels: kPrefix has one unit line per group of
// sequences, all of whose rows see all shared keys; kOwn has every sequence's keys behind them.  Both leave their results, whole or
// in pieces, in the workspace, with a reference per row that says where, and one kernel joins them.
#pragma once

#include "mq_kv.cuh"

namespace mq {

enum KvMode { kPlain, kPrefix, kOwn };

struct KvSchedArgs {
  KvBatchView b;
  int page_shift, max_q, n_kv;
  FastDiv group;   // query heads per key/value head
  FastDiv by_rows; // `rows` as a divisor
  int rows;        // query rows of a unit
  int pitch;       // rows between the slots of partial results (at least `rows`)
  int tile, tile_shift;   // keys of a tile (a power of two)
  int extra;       // a unit's cost besides its tiles, in tiles
  int min_len;     // a worker's range is at least this long (fewer workers for little work)
  const int32_t *leader, *shared_len;   // kPrefix, kOwn: of every sequence, the first of its group and the keys shared with it
};

// Keys [0, end) that row block rb of a sequence may see any of, and the tiles that hold them (at least one: a unit that
// sees nothing still has to write its zeros).  (Rows of a sequence, tokens x group, are below 2^30.)
template <KvMode kMode = kPlain>
__device__ __forceinline__ int sched_end(const KvSchedArgs& a, const KvSeq& s, int rb) {
  if (kMode == kPrefix || a.b.perm) return s.n_all;
  const int last = min((rb * a.rows + a.rows - 1) / a.group, s.n_new - 1);
  return max(0, min(s.n_all, s.n_all - s.n_new + last + 1));
}
template <KvMode kMode = kPlain>
__device__ __forceinline__ int sched_tiles(const KvSchedArgs& a, const KvSeq& s, int rb) {
  return max(1, (sched_end<kMode>(a, s, rb) + a.tile - 1) >> a.tile_shift);
}
__device__ __forceinline__ int sched_blocks(const KvSchedArgs& a, const KvSeq& s) {
  return (s.n_new * a.group.d + a.rows - 1) / a.by_rows;
}

// Shared memory of a sequence besides its place on the line: lengths, and for the lines of shared prefixes two numbers more
template <KvMode kMode>
constexpr int kSeqBytes = (int)sizeof(KvSeq) + (kMode == kPlain ? 0 : 8);
constexpr int kMaxSharedSeqs = 1024;   // sequences of a call with shared prefixes: all of them are held in shared memory

// What the groups share, and what follows from it for the line: seqs[b] becomes the group's rows and shared keys (kPrefix, at its
// first sequence; the others have no rows) or the sequence with its own keys only, which begin at page page0[b] of its list (kOwn).  A
// group shares whole pages, no more keys than any of its sequences with rows has cached, and nothing if it has fewer than two of
// those or its sequences do not stand side by side behind the first.  `prefix` is scratch here.
template <int kThreads, KvMode kMode>
__device__ __forceinline__ void sched_groups(const KvSchedArgs& a, int64_t* prefix, KvSeq* seqs, int* page0) {
  const int n = a.b.n_seq;
  int mine = -1;                                     // keys that this thread's first sequence can share (-1: it has no rows)
  int* keys = page0 + n;                             // of the group that begins at b
  int2* group = reinterpret_cast<int2*>(prefix);     // its sequences with rows, the last of them
  for (int b = threadIdx.x; b < n; b += kThreads) {  // (all loads at once; the leader waits in page0's place)
    const int l = a.leader[b], shared = a.shared_len[b];
    const KvSeq s = kv_seq(a.b, a.page_shift, a.max_q, b);
    seqs[b] = s;
    page0[b] = l;
    keys[b] = INT_MAX;
    group[b] = make_int2(0, b);
    if (b == threadIdx.x) mine = s.n_new > 0 ? max(0, min(shared, s.n_all - s.n_new)) : -1;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < n; b += kThreads) {
    const int l = page0[b];
    if (l < 0 || l > b) continue;
    // (rows in front of its neighbour's: a cu_q that decreases.  The group's rows are counted from the first one's to the last one's, which could be
    // fewer than none.)
    if (page0[l] != l || (l < b && (page0[b - 1] != l || seqs[b].begin < seqs[b - 1].begin))) {
      atomicMin(&keys[l], 0);
      continue;
    }
    if (b != threadIdx.x) {
      const KvSeq s = seqs[b];
      mine = s.n_new > 0 ? max(0, min(a.shared_len[b], s.n_all - s.n_new)) : -1;
    }
    if (mine >= 0) {
      atomicMin(&keys[l], mine);
      atomicAdd(&group[l].x, 1);
      atomicMax(&group[l].y, b);
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < n; b += kThreads) {
    const int l = page0[b];
    const int pages = l >= 0 && l <= b && group[l].x > 1 ? keys[l] >> a.page_shift : 0;
    page0[b] = kMode == kOwn ? pages : 0;
    if (kMode == kOwn) {
      seqs[b].n_all = max(0, seqs[b].n_all - (pages << a.page_shift));
    } else if (l == b && pages > 0) {
      const KvSeq last = kv_seq(a.b, a.page_shift, a.max_q, group[b].y);
      seqs[b].n_new = last.begin + last.n_new - seqs[b].begin;
      seqs[b].n_all = pages << a.page_shift;
    } else {
      seqs[b].n_new = 0;
    }
  }
  __syncthreads();
}

// prefix[b] = length of all units before sequence b; prefix[n_seq] = the whole line.  Called by every thread of a block of kThreads;
// `red` is shared scratch of kThreads / 32 entries.  `seqs`, if given, is shared memory that keeps the sequences' lengths for
// sched_unit (a dependent global load per unit costs about as much as a tile).
template <int kThreads, KvMode kMode = kPlain>
__device__ __forceinline__ void sched_prefix(const KvSchedArgs& a, int64_t* prefix, int64_t* red, KvSeq* seqs = nullptr, int* page0 = nullptr) {
  if (kMode != kPlain) sched_groups<kThreads, kMode>(a, prefix, seqs, page0);
  const int n = a.b.n_seq, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (n + kThreads - 1) / kThreads;
  int64_t sum = 0;
  for (int k = 0; k < per; ++k) {
    const int b = tid * per + k;
    if (b >= n) break;
    const KvSeq s = kMode != kPlain ? seqs[b] : kv_seq(a.b, a.page_shift, a.max_q, b);
    if (kMode == kPlain && seqs) seqs[b] = s;
    const int blocks = sched_blocks(a, s);
    int64_t t = 0;
    if (kMode == kPrefix || a.b.perm) t = (int64_t)blocks * (blocks ? sched_tiles<kMode>(a, s, 0) + a.extra : 0);
    else
      for (int rb = 0; rb < blocks; ++rb) t += sched_tiles(a, s, rb) + a.extra;
    sum += t * a.n_kv;
    prefix[b + 1] = sum;   // within this thread's run; the offset follows
  }
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) red[warp] = inc;
  __syncthreads();
  int64_t off = inc - sum;
  for (int w = 0; w < warp; ++w) off += red[w];
  for (int k = 0; k < per; ++k) {
    const int b = tid * per + k;
    if (b >= n) break;
    prefix[b + 1] += off;
  }
  if (tid == 0) prefix[0] = 0;
  __syncthreads();
}

// The unit that holds position `at` of the line; `skip` is the place in it (0 .. extra + tiles - 1).
struct KvUnit {
  int b, g, rb, tiles, skip;
  KvSeq s;
};
template <KvMode kMode = kPlain>
__device__ __forceinline__ KvUnit sched_unit(const KvSchedArgs& a, const int64_t* prefix, int64_t at, const KvSeq* seqs = nullptr) {
  int lo = 0, hi = a.b.n_seq;   // prefix[lo] <= at < prefix[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= at) lo = mid;
    else hi = mid;
  }
  KvUnit u;
  u.b = lo;
  u.s = seqs ? seqs[lo] : kv_seq(a.b, a.page_shift, a.max_q, lo);
  const int64_t all = prefix[lo + 1] - prefix[lo], x = at - prefix[lo];
  int64_t y;
  if (all >> 31) {
    const int64_t per_head = all / a.n_kv;
    u.g = (int)(x / per_head);
    y = x - u.g * per_head;
  } else {   // (the usual case, in 32 bits)
    const uint32_t per_head = (uint32_t)all / (uint32_t)a.n_kv;
    u.g = (int)((uint32_t)x / per_head);
    y = (uint32_t)x - (uint32_t)u.g * per_head;
  }
  u.tiles = sched_tiles<kMode>(a, u.s, 0);
  u.rb = 0;
  if (kMode == kPrefix || a.b.perm) {
    if (y >= u.tiles + a.extra) u.rb = (int)(y / (u.tiles + a.extra));
    y -= (int64_t)u.rb * (u.tiles + a.extra);
  } else {
    while (y >= u.tiles + a.extra) {
      y -= u.tiles + a.extra;
      u.tiles = sched_tiles(a, u.s, ++u.rb);
    }
  }
  u.skip = (int)y;
  return u;
}

// Length of a worker's range: the line cut into at most `grid` equal ranges (the last one may be shorter or empty).
__device__ __forceinline__ int64_t sched_share(const KvSchedArgs& a, int64_t total, int grid) {
  if (total <= (int64_t)grid * a.min_len) return a.min_len;
  return total >> 31 ? (total + grid - 1) / grid : (int64_t)(((uint32_t)total + (uint32_t)grid - 1u) / (uint32_t)grid);
}

// ---- partial results -----------------------------------------------------------------------------------
// Worker w has two slots: 2 w for a range's first piece when it starts inside a unit, 2 w + 1 for a piece that starts
// with its unit and does not reach its end.  Record w names the unit whose first piece is in slot 2 w + 1.
struct __align__(16) KvRecord {
  int n_parts;   // 0: this worker left no first piece; else the pieces are slots 2 w + 1, 2 (w + 1), 2 (w + 2), ...
  int begin;     // first row of the sequence in Q, O and lse
  int row0;      // the unit's first query row (token x group + head of the group) and how many it has
  int n_rows;
  int g;
  int pad[3];
};
struct KvParts {
  KvRecord* rec;   // [workers]
  float2* ml;      // [2 workers][pitch]: exponent reference (log2 units), sum
  float* o;        // [2 workers][pitch][D]
};
inline size_t kv_parts_bytes(int workers, int pitch, int dim) {
  return align_up((size_t)workers * sizeof(KvRecord), 256) + align_up((size_t)workers * 2 * pitch * sizeof(float2), 256) +
         (size_t)workers * 2 * pitch * dim * sizeof(float);
}
inline KvParts kv_parts(uint8_t* base, int workers, int pitch) {
  KvParts p;
  p.rec = reinterpret_cast<KvRecord*>(base);
  base += align_up((size_t)workers * sizeof(KvRecord), 256);
  p.ml = reinterpret_cast<float2*>(base);
  base += align_up((size_t)workers * 2 * pitch * sizeof(float2), 256);
  p.o = reinterpret_cast<float*>(base);
  return p;
}

struct KvOutArgs {
  __nv_bfloat16* O;
  int64_t ldo;
  float* lse;
  int n_q_heads;
};

// Results of the lines of shared prefixes, which the join turns into the output.  Row = token x query heads + head.
struct __align__(16) KvRowRef {
  int worker;    // its first piece is in slot 2 worker + 1, the next ones in 2 (worker + 1), ..
  int n_parts;   // 0: not in pieces, but in KvWhole; -1: the row belongs to no sequence
  int row;       // of a slot
  int more;      // kOwn: the row has a result over shared keys, too
};
struct KvWhole {
  KvRowRef* ref;     // [rows]
  KvRowRef* clear;   // kPrefix: the references of the other line, set to "no sequence" before it runs
  int64_t n_rows;
  float2* ml;        // [rows]
  float* o;          // [rows][D], unnormalised
};

// joins the pieces of split units
int launch_kv_combine(const KvSchedArgs& a, const KvParts& parts, const KvOutArgs& out, int workers, int dim, cudaStream_t st);

// the tensor-memory form for long chunks (mq_kv_chunk.cu)
struct KvAttnArgs {
  const uint8_t* Q;
  int64_t ldq;       // bytes
  KvSchedArgs sched;
  KvView cache;
  KvOutArgs out;
  KvParts parts;
  float scale;
  int32_t* status;
  KvWhole whole;     // kPrefix, kOwn
};

// How a call's work is divided: which kernel, its units, its workers
struct KvPlan {
  bool chunk;
  int workers, rows, pitch, tile, extra;
};
// n_lists lists of keys, each for at most max_q tokens
KvPlan kv_plan_attention(const mq_kv_batch* b, const mq_kv_cache* c, int group, int64_t n_lists, int64_t max_q);
void kv_set_plan(KvAttnArgs* a, const KvPlan& p, const mq_kv_cache* cache, int max_q, int group);
int launch_kv_lines(const KvAttnArgs& a, const KvPlan& p, KvMode mode, int dim, bool i8, cudaStream_t st);
int check_kv_attention(const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads, KvBatchView* bv, KvView* cv);

// The two lines run side by side: kOwn is launched behind kPrefix, but neither reads what the other writes, and where kPrefix leaves SMs idle
// kOwn begins at once.  For that kPrefix lets it start only when the kernel before both has completed (its own wait is over) and the
// references are cleared; kOwn then waits for nothing at its start, and at its end for kPrefix, so that the join, which waits for kOwn, has
// both.
template <KvMode kMode>
__device__ __forceinline__ void kv_begin(const KvWhole& w) {
  if (kMode == kPrefix) {
    pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < w.n_rows; i += (int64_t)gridDim.x * blockDim.x)
      w.clear[i] = KvRowRef{0, -1, 0, 0};
    __threadfence();
    __syncthreads();
    pdl_launch_dependents();
  } else {
    pdl_launch_dependents();
    if (kMode == kPlain) pdl_wait();
  }
}
template <KvMode kMode>
__device__ __forceinline__ void kv_end() {
  if (kMode == kOwn) pdl_wait();
}

void kv_chunk_shape(int group, int* rows, int* pitch, int* tile, int* extra);
int launch_kv_chunk(const KvAttnArgs& a, KvMode mode, int dim, bool i8, int workers, cudaStream_t st);

}  // namespace mq
