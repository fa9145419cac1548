// Accumulated softmax weights of the cached keys for chunks of many query rows, on the tensor cores (tcgen05).
//
//   sum over rows r of exp2(scale K Q^T - lse)[key, r],  one thread per key
//
// The transposed product: a unit is 128 keys of one (sequence, key/value head), the A operand; query rows come in tiles of up
// to 128 (whole tokens x the heads of the group) as the B operand.  With keys along the lanes of tensor memory a key's sum is
// a thread's own: it reads its scores, subtracts the columns' log-sum-exp (shared memory, the same address for all lanes),
// and adds exponentials; nothing is exchanged until the two groups of four warps, which take turns at the row tiles, add
// their sums at the unit's end.  Four score buffers fill tensor memory.  Every key is written once, in one order of
// summation.  Bound by the exponentials (128 x 128 of them cost the special-function pipe twice what the product costs
// the tensor pipe): chunks of 900 and 1024 tokens over 9092 and 3024 keys, 32 / 8 heads of 128 (85 GFLOP): 159 us, 115 without the
// exponentials, 99 for products and loads alone; 640 units over 148 CTAs are 5 for some and 4.3 on average.  All forms
// spill 24 to 28 bytes.
// A persistent CTA per SM takes the units whose start lies in its share of the line of all row tiles.
#include <cuda.h>

#include "mq_kv_tma.cuh"
#include "mq_kv_weights.cuh"

namespace mq {
namespace {

constexpr int kKeys = 128;              // keys of a unit
constexpr int kCols = 128;              // query rows of a tile
constexpr int kHalfBytes = 128 * 128;   // 128 rows x 64 bf16, swizzled
constexpr int kQStages = 4;
constexpr int kLStages = 8;
constexpr int kExtra = 1;               // a unit's cost besides its row tiles
constexpr int kRing = 8;

struct Piece {
  int live;               // 0: the line has ended
  int key0, n_all, ctx, n_rows;
  int tile0, tiles;       // row tiles
  int b, g, begin;
};

struct Barriers {
  uint64_t piece_full[kRing], piece_empty[kRing];
  uint64_t k_full[2], k_empty[2];
  uint64_t q_full[kQStages], q_empty[kQStages], l_full[kLStages], l_empty[kLStages];   // queries; their log-sum-exps
  uint64_t s_full[4], s_empty[4];
  uint64_t x_full[kRing];   // the second group's sums of a piece stand in shared memory
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
  int32_t status[2];   // as the waits leave it; passed on to the caller's words at the end
};

template <int kD, bool kI8>
struct Cfg {
  static constexpr int kHalves = kD / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kThreads = (kI8 ? 16 : 12) * 32;
  static constexpr int kSmem = 1024 + (2 + kQStages) * kTileBytes + (int)sizeof(Barriers) + kRing * (int)sizeof(Piece) + kLStages * kCols * 8 +
                               kRing * kKeys * 4 + 16 * 8 + 64;
};

// First row tile of the unit of keys key0 ..: without perm the rows before the first key's own see none of them.
__device__ __forceinline__ int first_tile(const WeightParams& p, const KvSeq& s, int tokens, int key0) {
  return p.b.perm ? 0 : max(0, key0 - (s.n_all - s.n_new)) / tokens;
}

// acc += exp2(score * scale - lse) of 32 columns
__device__ __forceinline__ void sum_cols(const uint32_t (&v)[32], const float* nl, float2 scale2, float2 (&acc)[2]) {
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    const float4 l = *reinterpret_cast<const float4*>(nl + e);
    const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), scale2, make_float2(l.x, l.y));
    const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), scale2, make_float2(l.z, l.w));
    acc[0] = __fadd2_rn(acc[0], make_float2(kv_exp2(x.x), kv_exp2(x.y)));
    acc[1] = __fadd2_rn(acc[1], make_float2(kv_exp2(y.x), kv_exp2(y.y)));
  }
}
// The same where a column counts only if lo <= its number < hi or, given ranks, if its rank is at least kp.
__device__ __forceinline__ void sum_cols_masked(const uint32_t (&v)[32], const float* nl, float2 scale2, float2 (&acc)[2], const int32_t* rk, int kp,
                                                int lo, int hi) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    const float2 l = *reinterpret_cast<const float2*>(nl + e);
    const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), scale2, l);
    const bool p0 = rk ? kp <= rk[e] : e >= lo && e < hi, p1 = rk ? kp <= rk[e + 1] : e + 1 >= lo && e + 1 < hi;
    acc[0] = __fadd2_rn(acc[0], make_float2(p0 ? kv_exp2(x.x) : 0.0f, p1 ? kv_exp2(x.y) : 0.0f));
  }
}

template <int kD, bool kI8>
__global__ void __launch_bounds__(Cfg<kD, kI8>::kThreads, 1)
kv_weights_chunk_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                        const __grid_constant__ WeightParams p) {
  using C = Cfg<kD, kI8>;
  constexpr int kTileBytes = C::kTileBytes, kHalves = C::kHalves;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* k_smem = smem;                              // two buffers
  uint8_t* q_smem = k_smem + 2 * kTileBytes;
  Barriers* sh = reinterpret_cast<Barriers*>(q_smem + kQStages * kTileBytes);
  Piece* ring = reinterpret_cast<Piece*>(sh + 1);
  float* neg_lse = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(ring + kRing) + 15) & ~uintptr_t(15));   // [stage][col], log2 units
  int32_t* rank = reinterpret_cast<int32_t*>(neg_lse + kLStages * kCols);                                        // [stage][col]
  float* xch = reinterpret_cast<float*>(rank + kLStages * kCols);                                                // [piece][key]
  int64_t* red = reinterpret_cast<int64_t*>(xch + kRing * kKeys);
  int64_t* prefix = red + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
  const int tokens = kCols / p.group, block_rows = tokens * p.group.d;

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_q)) : "memory");
    if (!kI8) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_k)) : "memory");
    for (int i = 0; i < kRing; ++i) { mbar_init(&sh->piece_full[i], 1); mbar_init(&sh->piece_empty[i], 8); mbar_init(&sh->x_full[i], 4); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh->k_full[i], kI8 ? 4 : 1); mbar_init(&sh->k_empty[i], 1); }
    for (int i = 0; i < kQStages; ++i) { mbar_init(&sh->q_full[i], 1); mbar_init(&sh->q_empty[i], 1); }
    for (int i = 0; i < kLStages; ++i) { mbar_init(&sh->l_full[i], 1); mbar_init(&sh->l_empty[i], 4); }
    for (int i = 0; i < 4; ++i) { mbar_init(&sh->s_full[i], 1); mbar_init(&sh->s_empty[i], 4); }
    mbar_init(&sh->drain, 1);
    sh->abort_flag = 0;
    sh->status[0] = sh->status[1] = MQ_OK;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a query tile that no box fills (a group that does not divide 128): zeros, so that their scores are finite
  for (int i = tid; i < kQStages * kHalves * (kCols - block_rows) * 8; i += C::kThreads) {
    const int per = (kCols - block_rows) * 8, blk = i / per, r = block_rows + (i % per) / 8;
    *reinterpret_cast<uint4*>(q_smem + blk * kHalfBytes + r * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async_smem();
  if (warp == 2) {
    tmem_alloc(&sh->tmem_base, 512);
    tmem_relinquish();
  }
  pdl_launch_dependents();
  pdl_wait();
  tc_fence_before();

  // ---- the line: per sequence, head and 128 keys, the row tiles plus kExtra
  const int n = p.b.n_seq;
  {
    const int per = (n + C::kThreads - 1) / C::kThreads;
    int64_t sum = 0;
    for (int k = 0; k < per; ++k) {
      const int b = tid * per + k;
      if (b >= n) break;
      const KvSeq s = kv_seq(p.b, p.c.page_shift, p.max_q, b);
      const int blocks = (s.n_all + kKeys - 1) / kKeys, nt = (s.n_new + tokens - 1) / tokens, ctx = s.n_all - s.n_new;
      // blocks that start inside the context meet every row tile
      const int full = p.b.perm ? blocks : min(blocks, ctx < 0 ? 0 : ctx / kKeys + 1);
      int64_t t = (int64_t)full * (max(nt, 1) + kExtra);
      for (int kb = full; kb < blocks; ++kb) t += max(nt - first_tile(p, s, tokens, kb * kKeys), 1) + kExtra;
      sum += t * p.c.n_kv_heads;
      prefix[b + 1] = sum;
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
  tc_fence_after();
  const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh->tmem_base);

  auto get_piece = [&](int np, bool& ok, int site) -> const Piece* {
    ok = mbar_wait(&sh->piece_full[np % kRing], (uint32_t)(np / kRing) & 1u, &sh->abort_flag, sh->status, site);
    if (!ok) return nullptr;
    const Piece* pc = ring + np % kRing;
    return pc->live ? pc : nullptr;
  };

  if (!kI8 && warp == 0) {
    // ---------------- the unit's keys by TMA: lane i brings page i of the 128 keys
    const int shift = p.c.page_shift, rows = shift >= 7 ? kKeys : 1 << shift, boxes = kKeys / rows;
    bool ok = true;
    int np = 0;
    for (; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 70);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int buf = np & 1, key = pc->key0 + lane * rows;
      int page = max(p.c.n_pages, 1);   // a page number the map does not have: zeros
      if (lane < boxes && key < pc->n_all) {
        const int pg = p.b.page_table[(int64_t)pc->b * p.b.max_pages + (key >> shift)];
        if ((unsigned)pg < (unsigned)p.c.n_pages) page = pg;
        else if (p.status) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
      }
      if (np >= 2 && !(ok = warp_all(mbar_wait(&sh->k_empty[buf], (uint32_t)(np / 2 - 1) & 1u, &sh->abort_flag, sh->status, 71)))) break;
      if (lane == 0) mbar_arrive_expect_tx(&sh->k_full[buf], kTileBytes);
      __syncwarp();
      if (lane < boxes) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
          tma_load_4d(smem_u32(k_smem + buf * kTileBytes + h * kHalfBytes + lane * rows * 128), &tmap_k, h * 64, key & ((1 << shift) - 1), pc->g, page,
                      &sh->k_full[buf]);
      }
      __syncwarp();
    }
    if (!ok)
      for (int back = 1; back <= 2 && back <= np; ++back) mbar_wait_drain(&sh->k_full[(np - back) & 1], (uint32_t)((np - back) / 2) & 1u, 20000ull);
  } else if (warp == 1) {
    // ---------------- MMA issuer
    if (elect_one()) {
      const uint32_t idesc = make_idesc_bf16(kCols);
      bool ok = true;
      int t = 0;
      for (int np = 0;; ++np) {
        const Piece* pc = get_piece(np, ok, 72);
        if (!pc) break;
        const int tiles = pc->tiles, buf = np & 1;
        if (!(ok = mbar_wait(&sh->k_full[buf], (uint32_t)(np / 2) & 1u, &sh->abort_flag, sh->status, 73))) break;
        const uint64_t kdesc = make_b_desc(smem_u32(k_smem + buf * kTileBytes));
        for (int i = 0; i < tiles; ++i, ++t) {
          const int qs = t % kQStages, sb = t & 3;
          if (!(ok = mbar_wait(&sh->q_full[qs], (uint32_t)(t / kQStages) & 1u, &sh->abort_flag, sh->status, 74))) break;
          if (t >= 4 && !(ok = mbar_wait(&sh->s_empty[sb], (uint32_t)(t / 4 - 1) & 1u, &sh->abort_flag, sh->status, 75))) break;
          tc_fence_after();
          const uint64_t qdesc = make_b_desc(smem_u32(q_smem + qs * kTileBytes));
#pragma unroll
          for (int k = 0; k < kD / 16; ++k) {
            const uint64_t off = (uint64_t)((k >> 2) * (kHalfBytes >> 4) + (k & 3) * 2);
            mma_bf16_ss(tmem_base + (uint32_t)(sb * kCols), kdesc + off, qdesc + off, idesc, k ? 1u : 0u);
          }
          tc_commit(&sh->s_full[sb]);
          tc_commit(&sh->q_empty[qs]);
        }
        if (!ok) break;
        tc_commit(&sh->k_empty[buf]);
      }
      if (!ok) {
        tc_commit(&sh->drain);
        mbar_wait_drain(&sh->drain, 0, 2000000ull);
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---------------- walks the line, publishes the units, brings their queries
    const int64_t total = prefix[n], share = (total + gridDim.x - 1) / gridDim.x;
    const int64_t lo = min(total, (int64_t)blockIdx.x * share), hi = min(total, lo + share);
    bool ok = true;
    int t = 0, np = 0;
    // the first unit that starts at or behind lo
    int b = 0, g = 0, kb = 0;
    int64_t at = hi;   // (a worker whose share is empty)
    KvSeq s{};
    int nt = 0, blocks = 0;
    if (lo < hi) {
      int x = 0, y = n;
      while (y - x > 1) {
        const int mid = (x + y) >> 1;
        if (prefix[mid] <= lo) x = mid;
        else y = mid;
      }
      b = x;
      s = kv_seq(p.b, p.c.page_shift, p.max_q, b);
      nt = (s.n_new + tokens - 1) / tokens;
      blocks = (s.n_all + kKeys - 1) / kKeys;
      const int64_t per_head = (prefix[b + 1] - prefix[b]) / p.c.n_kv_heads;
      g = (int)((lo - prefix[b]) / per_head);
      at = prefix[b] + g * per_head;
      // (the units that meet every row tile are alike)
      const int full = p.b.perm ? blocks : min(blocks, s.n_all - s.n_new < 0 ? 0 : (s.n_all - s.n_new) / kKeys + 1);
      const int64_t each = max(nt, 1) + kExtra, need = (lo - at + each - 1) / each;
      kb = (int)(need < full ? need : full);
      at += kb * each;
      if (kb == blocks) { kb = 0; ++g; }
      while (at < lo) {
        at += max(nt - first_tile(p, s, tokens, kb * kKeys), 1) + kExtra;
        if (++kb == blocks) { kb = 0; ++g; }
      }
    }
    while (ok) {
      Piece pc{};
      if (at < hi) {
        while (kb >= blocks || g >= p.c.n_kv_heads) {   // the next sequence that has keys (there is one: at < total)
          s = kv_seq(p.b, p.c.page_shift, p.max_q, ++b);
          nt = (s.n_new + tokens - 1) / tokens;
          blocks = (s.n_all + kKeys - 1) / kKeys;
          g = kb = 0;
        }
        pc.live = 1;
        pc.key0 = kb * kKeys;
        pc.n_all = s.n_all;
        pc.ctx = s.n_all - s.n_new;
        pc.n_rows = s.n_new * p.group.d;
        pc.tile0 = first_tile(p, s, tokens, pc.key0);
        pc.tiles = max(nt - pc.tile0, 1);
        pc.b = b;
        pc.g = g;
        pc.begin = s.begin;
        at += pc.tiles + kExtra;
        if (++kb == blocks) { kb = 0; ++g; }
      }
      if (np >= kRing && !(ok = warp_all(mbar_wait(&sh->piece_empty[np % kRing], (uint32_t)(np / kRing - 1) & 1u, &sh->abort_flag, sh->status, 76)))) break;
      if (lane == 0) {
        ring[np % kRing] = pc;
        mbar_arrive(&sh->piece_full[np % kRing]);
      }
      __syncwarp();
      if (!pc.live) break;
      for (int i = 0; i < pc.tiles; ++i, ++t) {
        const int qs = t % kQStages;
        if (t >= kQStages && !(ok = warp_all(mbar_wait(&sh->q_empty[qs], (uint32_t)(t / kQStages - 1) & 1u, &sh->abort_flag, sh->status, 77)))) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&sh->q_full[qs], (uint32_t)(block_rows * 128 * kHalves));
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_3d(smem_u32(q_smem + qs * kTileBytes + h * kHalfBytes), &tmap_q, h * 64, pc.g * p.group.d, pc.begin + (pc.tile0 + i) * tokens, &sh->q_full[qs]);
        }
        __syncwarp();
      }
      ++np;
    }
    if (!ok)
      for (int back = 1; back <= kQStages && back <= t; ++back)
        mbar_wait_drain(&sh->q_full[(t - back) % kQStages], (uint32_t)((t - back) / kQStages) & 1u, 20000ull);
  } else if (warp == 3) {
    // ---------------- the rows' log-sum-exps (negated, log2 units; -inf where a column adds nothing) and ranks
    bool ok = true;
    int t = 0;
    int tok_of[4], head_of[4];   // of this lane's columns, within a tile
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      tok_of[c] = (c * 32 + lane) / p.group;
      head_of[c] = (c * 32 + lane) - tok_of[c] * p.group.d;
    }
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 78);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int tiles = pc->tiles, tile0 = pc->tile0, n_rows = pc->n_rows, begin = pc->begin, g_head = pc->g * p.group.d;
      float l_next[4];
      int rk_next[4];
      auto fetch = [&](int i) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int col = c * 32 + lane;
          l_next[c] = INFINITY;
          rk_next[c] = INT_MIN;
          if (i < tiles && col < block_rows && (tile0 + i) * block_rows + col < n_rows) {
            const int tok = begin + (tile0 + i) * tokens + tok_of[c];
            l_next[c] = p.lse[(int64_t)tok * p.n_q_heads + g_head + head_of[c]];
            rk_next[c] = p.b.perm ? p.b.perm[tok] : 0;
          }
        }
      };
      fetch(0);
      for (int i = 0; i < tiles; ++i, ++t) {
        const int ls = t % kLStages;
        float l[4];
        int rk[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) { l[c] = l_next[c]; rk[c] = rk_next[c]; }
        fetch(i + 1);   // the next tile's are on their way while this one's slot is waited for
        if (t >= kLStages && !(ok = warp_all(mbar_wait(&sh->l_empty[ls], (uint32_t)(t / kLStages - 1) & 1u, &sh->abort_flag, sh->status, 79)))) break;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          // (the log-sum-exp of a row that sees nothing is -inf: it adds nothing either)
          neg_lse[ls * kCols + c * 32 + lane] = fabsf(l[c]) == INFINITY ? -INFINITY : l[c] * -1.4426950408889634f;
          rank[ls * kCols + c * 32 + lane] = rk[c];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->l_full[ls]);
      }
    }
  } else if (warp >= 4 && warp < 12) {
    // ---------------- sums: group grp takes the row tiles of its parity; a thread owns one key
    const int quarter = warp & 3, grp = (warp - 4) >> 2, r = quarter * 32 + lane;
    const uint32_t lane_base = tmem_base + ((uint32_t)(quarter * 32) << 16);
    bool ok = true;
    int t = 0;
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 80);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int key = pc->key0 + r, ctx = pc->ctx, n_all = pc->n_all, tiles = pc->tiles, tile0 = pc->tile0, n_rows = pc->n_rows;
      const int32_t* perm = p.b.perm ? p.b.perm + pc->begin : nullptr;
      const int kp = key >= n_all ? INT_MAX : key < ctx ? -1 : perm ? perm[key - ctx] : 0;
      const float scale_log2 = p.scale * 1.4426950408889634f * (kI8 ? p.c.k_scale[pc->g] : 1.0f);
      const float2 scale2 = make_float2(scale_log2, scale_log2);
      const int64_t out = (int64_t)pc->b * p.seq_stride + (int64_t)pc->g * p.head_stride + key;
      float sum = 0.0f;
      for (int i = 0; i < tiles && ok; ++i, ++t) {
        if ((t & 1) != grp) continue;
        const int ls = t % kLStages, sb = t & 3, row0 = (tile0 + i) * block_rows;
        // rows not seen in full by all keys of the unit, or columns behind the last row
        const bool masked = row0 + block_rows > n_rows || (perm ? pc->key0 + kKeys > ctx : (tile0 + i) * tokens < pc->key0 + kKeys - 1 - ctx);
        if (!(ok = warp_all(mbar_wait(&sh->l_full[ls], (uint32_t)(t / kLStages) & 1u, &sh->abort_flag, sh->status, 81)))) break;
        if (!(ok = warp_all(mbar_wait(&sh->s_full[sb], (uint32_t)(t / 4) & 1u, &sh->abort_flag, sh->status, 82)))) break;
        tc_fence_after();
        // columns lo .. hi - 1 count (without perm); with it, columns whose rank is at least kp
        const int lo = perm ? 0 : (int)max((int64_t)0, min((int64_t)kCols, (int64_t)(key - ctx) * p.group.d - row0)), hi = n_rows - row0;
        float2 acc[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        const uint32_t s_addr = lane_base + (uint32_t)(sb * kCols);
        uint32_t va[32], vb[32];   // the next 32 columns are on their way while these are summed
        tmem_ld_x32(s_addr, va);
        tmem_wait_ld();
        tmem_ld_x32(s_addr + 32u, vb);
        if (!masked) {
          sum_cols(va, neg_lse + ls * kCols, scale2, acc);
          tmem_wait_ld();
          tmem_ld_x32(s_addr + 64u, va);
          sum_cols(vb, neg_lse + ls * kCols + 32, scale2, acc);
          tmem_wait_ld();
          tmem_ld_x32(s_addr + 96u, vb);
          sum_cols(va, neg_lse + ls * kCols + 64, scale2, acc);
          tmem_wait_ld();
          sum_cols(vb, neg_lse + ls * kCols + 96, scale2, acc);
        } else {
          const int32_t* rk = perm ? rank + ls * kCols : nullptr;
          sum_cols_masked(va, neg_lse + ls * kCols, scale2, acc, rk, kp, lo, hi);
          tmem_wait_ld();
          tmem_ld_x32(s_addr + 64u, va);
          sum_cols_masked(vb, neg_lse + ls * kCols + 32, scale2, acc, rk ? rk + 32 : rk, kp, lo - 32, hi - 32);
          tmem_wait_ld();
          tmem_ld_x32(s_addr + 96u, vb);
          sum_cols_masked(va, neg_lse + ls * kCols + 64, scale2, acc, rk ? rk + 64 : rk, kp, lo - 64, hi - 64);
          tmem_wait_ld();
          sum_cols_masked(vb, neg_lse + ls * kCols + 96, scale2, acc, rk ? rk + 96 : rk, kp, lo - 96, hi - 96);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh->s_empty[sb]);
          mbar_arrive(&sh->l_empty[ls]);
        }
        sum += (acc[0].x + acc[0].y) + (acc[1].x + acc[1].y);
      }
      if (!ok) break;
      // ---- the unit's sums: the second group's first through shared memory, a slot per published piece (it is written again only
      // after both groups were done with its piece).  A bounded wait like all others: where one group has given up, the other
      // must not stay at a barrier for it.
      if (grp == 1) {
        xch[np % kRing * kKeys + r] = sum;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->x_full[np % kRing]);
      } else if (!(ok = warp_all(mbar_wait(&sh->x_full[np % kRing], (uint32_t)(np / kRing) & 1u, &sh->abort_flag, sh->status, 85)))) {
        break;
      }
      if (grp == 0 && key < n_all) {
        if (key < p.w_keys) p.W_out[out] = (p.W_in && key < ctx ? p.W_in[out] : 0.0f) + (sum + xch[np % kRing * kKeys + r]);
        else if (p.status) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->piece_empty[np % kRing]);
    }
  } else if (kI8 && warp >= 12) {
    // ---------------- int8 cache: the unit's keys widened to bf16, one key per thread
    const int r = (warp - 12) * 32 + lane, shift = p.c.page_shift;
    constexpr int kLoads = kD / 16;
    bool ok = true;
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 83);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int buf = np & 1, key = pc->key0 + r;
      uint4 x[kLoads];
#pragma unroll
      for (int c = 0; c < kLoads; ++c) x[c] = make_uint4(0u, 0u, 0u, 0u);
      if (key < pc->n_all) {
        const int pg = p.b.page_table[(int64_t)pc->b * p.b.max_pages + (key >> shift)];
        if ((unsigned)pg < (unsigned)p.c.n_pages) {
          const uint8_t* src = p.c.K + (int64_t)pg * p.c.page_stride + (int64_t)pc->g * p.c.head_stride + (int64_t)(key & ((1 << shift) - 1)) * p.c.slot_stride;
#pragma unroll
          for (int c = 0; c < kLoads; ++c) x[c] = *reinterpret_cast<const uint4*>(src + c * 16);
        } else if (p.status) {
          atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
        }
      }
      if (np >= 2 && !(ok = warp_all(mbar_wait(&sh->k_empty[buf], (uint32_t)(np / 2 - 1) & 1u, &sh->abort_flag, sh->status, 84)))) break;
      uint8_t* kd = k_smem + buf * kTileBytes + r * 128;
#pragma unroll
      for (int c = 0; c < kLoads; ++c) {
        uint4 a, b;
        i8x4_to_bf16(x[c].x, a.x, a.y); i8x4_to_bf16(x[c].y, a.z, a.w);
        i8x4_to_bf16(x[c].z, b.x, b.y); i8x4_to_bf16(x[c].w, b.z, b.w);
        uint8_t* blk = kd + (c >> 2) * kHalfBytes;
        *reinterpret_cast<uint4*>(blk + ((((2 * c) & 7) ^ (r & 7)) << 4)) = a;
        *reinterpret_cast<uint4*>(blk + ((((2 * c + 1) & 7) ^ (r & 7)) << 4)) = b;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->k_full[buf]);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (tid == 0 && sh->status[0] != MQ_OK && p.status && atomicCAS(p.status, MQ_OK, sh->status[0]) == MQ_OK) p.status[1] = sh->status[1];
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int kD, bool kI8>
int launch(const WeightParams& p, int64_t most, cudaStream_t st) {
  using C = Cfg<kD, kI8>;
  static_assert(C::kSmem + (kMaxKvSeqs + 1) * 8 <= 232448, "shared memory of one CTA");
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_weights_chunk_kernel<kD, kI8>, C::kSmem + (kMaxKvSeqs + 1) * (int)sizeof(int64_t))) return MQ_ERR_CUDA;
  CUtensorMap mq_{}, mk{};
  if (!encode_queries(&mq_, p.Q, p.ldq, p.n_q_heads, p.b.total_q, p.group.d, kCols / p.group.d * p.group.d, kD)) return MQ_ERR_CUDA;
  if (!kI8 && !encode_pages(&mk, p.c.K, p.Q, p.c, kD, kKeys)) return MQ_ERR_CUDA;
  const int64_t cap = sm_count();
  const cudaError_t e = launch_pdl(kv_weights_chunk_kernel<kD, kI8>, dim3((unsigned)(most < cap ? most : cap)), dim3(C::kThreads),
                                   C::kSmem + ((size_t)p.b.n_seq + 1) * sizeof(int64_t), st, mq_, mk, p);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace

int launch_kv_weights_chunk(const WeightParams& p, int dim, bool i8, int64_t most_units, cudaStream_t st) {
  if (dim == 128) return i8 ? launch<128, true>(p, most_units, st) : launch<128, false>(p, most_units, st);
  return i8 ? launch<64, true>(p, most_units, st) : launch<64, false>(p, most_units, st);
}

}  // namespace mq
