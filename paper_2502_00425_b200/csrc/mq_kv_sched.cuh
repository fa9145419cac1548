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
#pragma once

#include "mq_kv.cuh"

namespace mq {

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
};

// Keys [0, end) that row block rb of a sequence may see any of, and the tiles that hold them (at least one: a unit that
// sees nothing still has to write its zeros).  (Rows of a sequence, tokens x group, are below 2^30.)
__device__ __forceinline__ int sched_end(const KvSchedArgs& a, const KvSeq& s, int rb) {
  if (a.b.perm) return s.n_all;
  const int last = min((rb * a.rows + a.rows - 1) / a.group, s.n_new - 1);
  return max(0, min(s.n_all, s.n_all - s.n_new + last + 1));
}
__device__ __forceinline__ int sched_tiles(const KvSchedArgs& a, const KvSeq& s, int rb) {
  return max(1, (sched_end(a, s, rb) + a.tile - 1) >> a.tile_shift);
}
__device__ __forceinline__ int sched_blocks(const KvSchedArgs& a, const KvSeq& s) {
  return (s.n_new * a.group.d + a.rows - 1) / a.by_rows;
}

// prefix[b] = length of all units before sequence b; prefix[n_seq] = the whole line.  Called by every thread of a block of kThreads;
// `red` is shared scratch of kThreads / 32 entries.  `seqs`, if given, is shared memory that keeps the sequences' lengths for
// sched_unit (a dependent global load per unit costs about as much as a tile).
template <int kThreads>
__device__ __forceinline__ void sched_prefix(const KvSchedArgs& a, int64_t* prefix, int64_t* red, KvSeq* seqs = nullptr) {
  const int n = a.b.n_seq, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (n + kThreads - 1) / kThreads;
  int64_t sum = 0;
  for (int k = 0; k < per; ++k) {
    const int b = tid * per + k;
    if (b >= n) break;
    const KvSeq s = kv_seq(a.b, a.page_shift, a.max_q, b);
    if (seqs) seqs[b] = s;
    const int blocks = sched_blocks(a, s);
    int64_t t = 0;
    if (a.b.perm) t = (int64_t)blocks * (blocks ? sched_tiles(a, s, 0) + a.extra : 0);
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
  u.tiles = sched_tiles(a, u.s, 0);
  u.rb = 0;
  if (a.b.perm) {
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
};

void kv_chunk_shape(int group, int* rows, int* pitch, int* tile, int* extra);
int launch_kv_chunk(const KvAttnArgs& a, int dim, bool i8, int workers, cudaStream_t st);

}  // namespace mq
