// Attention of long chunks over a paged key/value cache on the tensor cores (tcgen05), for units of up to 256 query rows.
//
// The work line, units and partial results are those of mq_kv_sched.cuh; one persistent CTA per SM walks its range of the
// line.  A row of a unit is (token, query head of the group), so every key tile serves the whole group.
//   S = Q K^T (128 rows x 128 keys, bf16, float32 accumulators in tensor memory);  P = exp2(scale (S - ref));  O += P V
//   * A unit is two blocks of 128 rows (whole tokens), one for each of two groups of four softmax warps; both use every K and V
//     tile, which halves what a tile costs to bring and keeps the tensor pipe busy with one block while the other is in its
//     softmax.  Tensor memory is full: scores 2 x 128 columns, outputs 2 x 128.  A thread owns one row and works on its 128
//     scores in two steps of 64; P replaces the scores it was made from (it never leaves tensor memory), and the product of the
//     first 64 keys starts while the second 64 are still exponentials.  A unit of at most one block leaves the other group idle.
//   * K and V tiles (128 keys) come straight from the pages by TMA: one box per page and 64 channels, 128-byte swizzle, the
//     page number as the outermost coordinate; what lies behind the last key is asked for at a page number outside the map
//     and arrives as zeros.  V is the second product's B operand as it lies (channels contiguous), no transpose.  Queries
//     come as one box of (tokens x heads of the group) per 64 channels.
//   * An int8 cache is read by four more warps, which widen the codes exactly (K to bf16, V to fp16) into the same tiles.
//   * Tiles are numbered through over all units of a worker, so the products of the next unit's first tile are under way while
//     the softmax warps still write out the last unit.  One warp walks the work line and publishes its pieces to all roles.
//   * The exponents' reference may lag a row's maximum by 2^8 before the accumulator is rescaled.
// Visibility: a tile some row may not see in full is masked element by element, all others take no mask.  A value that some
// rows may not see must not reach them even if it is infinite or NaN: one warp looks through the value tiles that are not
// seen by all rows, replaces such values by zero before the product, and the rows that do see them get them at the end.
// The probabilities are rounded once, to the type of the value tiles (bf16, or fp16 over an int8 cache): a product of two types is not
// to be had, and float32 or a second term would double that product, on the pipe that is the bound.
// 2048 tokens behind 32768 keys, 28 / 4 heads of 128 (992 GFLOP): 825 us in a short run, 1.2 PFLOP/s (72 % of the measured GEMM
// rate), and 960 to 990 us in a long one, under the power cap.  A tile of 256 rows takes some 3700 cycles: 2 x 1300 of softmax per group, the rest the products that the
// two groups cannot hide for one another; the products alone would take 661 us, the softmax without exponentials 764.  Over an int8
// cache 16 warps share the registers, 128 a thread, which spills 80 bytes (with a shared prefix 120 - 128 on its line, 252 on the other).  Six turns of 40 to 701 tokens in AIFS order: 83 us, of which 51 at this rate.  A call of a few tiles is 5 us of start (work line, page
// table, first tiles), its tiles, 2 us of results and the join.
// Every wait is bounded (mq_sm100.cuh); an expired one makes all roles leave and sets the status word.
#include <cuda.h>

#include <cfloat>

#include "mq_kv_sched.cuh"
#include "mq_kv_tma.cuh"

namespace mq {
namespace {

constexpr int kBlock = 128;             // query rows of a block (one tensor-memory accumulator)
constexpr int kPitch = 2 * kBlock;      // rows of a partial result's slot
constexpr int kTile = 128;              // keys of a tile
constexpr int kHalfBytes = 128 * 128;   // 128 rows x 64 bf16, swizzled
constexpr int kStages = 2;
constexpr int kExtraTiles = 2;          // what a unit costs besides its tiles, in tiles
constexpr uint32_t kColO = 256;         // tensor memory: scores at 128 g, outputs at 256 + 128 g
constexpr float kLag = 8.0f;            // log2 of how far a row's maximum may outgrow the reference
// fp16 probabilities (int8 cache): the reference lies 6 below the maximum, so they run to 2^6, and to 2^14 with the lag
constexpr float kLiftChunk = 6.0f;
constexpr int kRing = 8;                // published pieces
constexpr int kSeqsHeld = 512;          // up to so many sequences have their lengths in shared memory (of a bf16 tile's 200 KB, 27 are left)

// v[k] of lane q of four neighbours <-> v[q] of lane k
__device__ __forceinline__ void quad_transpose(uint4 (&v)[4], int lane) {
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k & o) continue;
      uint4 x = up ? v[k] : v[k | o];
      x.x = __shfl_xor_sync(0xffffffffu, x.x, o);
      x.y = __shfl_xor_sync(0xffffffffu, x.y, o);
      x.z = __shfl_xor_sync(0xffffffffu, x.z, o);
      x.w = __shfl_xor_sync(0xffffffffu, x.w, o);
      if (up) v[k] = x;
      else v[k | o] = x;
    }
  }
}

// What a worker does next on the line: tiles t0 .. t1 - 1 of a unit (t0 == t1: the line's end).
struct Piece {
  int t0, t1, end, ctx;
  int row0, n_rows;       // query rows of the unit
  int all_see;            // every row of the unit sees the keys below
  const int32_t* table;   // page of the piece's first key
  int g, begin;
  int more;               // kOwn: the rows see shared keys, too
  int whole;              // the piece is the whole unit
  int n_parts;            // of the unit, if this is its first piece
  int poison;             // values were taken out of its tiles
};

struct ChunkBarriers {
  uint64_t piece_full[kRing], piece_empty[kRing];   // published; the eight softmax warps are done with it
  uint64_t q_full[2], q_empty[2];              // per block
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_ok[kStages], v_empty[kStages];
  uint64_t s_full[2], p_full[4], pv_done[4];   // [group], [2 group + step]
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
};

template <int kD, bool kI8>
struct ChunkCfg {
  static constexpr int kHalves = kD / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kThreads = (kI8 ? 16 : 12) * 32;
  static constexpr int kSmem = 1024 + (2 + 2 * kStages) * kTileBytes + (int)sizeof(ChunkBarriers) + kRing * (int)sizeof(Piece) + 8 * kTile * 4 + 16 * 8;
};

// B operand whose N (64 channels per block, 128-byte swizzle) is contiguous: blocks `block_bytes` apart, 8-key groups 1024 apart
__device__ __forceinline__ uint64_t desc_n_major(uint32_t addr, uint32_t block_bytes) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(block_bytes >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

template <int kD, bool kI8, KvMode kMode>
__global__ void __launch_bounds__(ChunkCfg<kD, kI8>::kThreads, 1)
kv_chunk_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ KvAttnArgs p) {
  using C = ChunkCfg<kD, kI8>;
  constexpr int kTileBytes = C::kTileBytes, kHalves = C::kHalves;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_smem = smem;                              // two blocks
  uint8_t* k_smem = q_smem + 2 * kTileBytes;
  uint8_t* v_smem = k_smem + kStages * kTileBytes;
  ChunkBarriers* sh = reinterpret_cast<ChunkBarriers*>(v_smem + kStages * kTileBytes);
  Piece* ring = reinterpret_cast<Piece*>(sh + 1);
  int32_t* kp_all = reinterpret_cast<int32_t*>(ring + kRing);   // [8 warps][128]
  int64_t* red = reinterpret_cast<int64_t*>(kp_all + 8 * kTile);
  int64_t* prefix = red + 16;
  KvSeq* seqs = kMode != kPlain || p.sched.b.n_seq <= kSeqsHeld ? reinterpret_cast<KvSeq*>(prefix + p.sched.b.n_seq + 1) : nullptr;
  int* page0 = reinterpret_cast<int*>(seqs + p.sched.b.n_seq);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_q)) : "memory");
    if (!kI8) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_k)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_v)) : "memory");
    }
    const uint32_t fills = kI8 ? 4 : 1;   // who fills a tile: one TMA thread, or four widening warps
    for (int i = 0; i < kRing; ++i) { mbar_init(&sh->piece_full[i], 1); mbar_init(&sh->piece_empty[i], 8); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh->q_full[i], 1); mbar_init(&sh->q_empty[i], 1); mbar_init(&sh->s_full[i], 1); }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh->k_full[i], fills); mbar_init(&sh->k_empty[i], 1);
      mbar_init(&sh->v_full[i], fills); mbar_init(&sh->v_ok[i], 1); mbar_init(&sh->v_empty[i], 1);
    }
    for (int i = 0; i < 4; ++i) { mbar_init(&sh->p_full[i], 4); mbar_init(&sh->pv_done[i], 1); }
    mbar_init(&sh->drain, 1);
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a query block that no box fills (a group that does not divide 128): zeros, not what the last kernel left there
  const int unfilled = kBlock - (p.sched.rows >> 1);
  for (int i = threadIdx.x; i < 2 * kHalves * unfilled * 8; i += C::kThreads) {
    const int blk = i / (unfilled * 8), r = kBlock - unfilled + (i % (unfilled * 8)) / 8;
    *reinterpret_cast<uint4*>(q_smem + blk * kHalfBytes + r * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async_smem();
  if (warp == 2) {
    tmem_alloc(&sh->tmem_base, 512);
    tmem_relinquish();
  }
  kv_begin<kMode>(p.whole);
  const KvSchedArgs& sc = p.sched;
  tc_fence_before();
  sched_prefix<C::kThreads, kMode>(sc, prefix, red, seqs, page0);   // (ends with __syncthreads)
  tc_fence_after();
  const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh->tmem_base);
  const int block_rows = sc.rows >> 1;          // rows of a block: whole tokens

  // The np-th piece, once published; false: the line has ended, or a wait expired (ok then says which).
  auto get_piece = [&](int np, bool& ok, int site) -> const Piece* {
    ok = mbar_wait(&sh->piece_full[np % kRing], (uint32_t)(np / kRing) & 1u, &sh->abort_flag, p.status, site);
    if (!ok) return nullptr;
    const Piece* pc = ring + np % kRing;
    return pc->t0 < pc->t1 ? pc : nullptr;
  };

  if (!kI8 && warp == 0) {
    // ---------------- TMA producer.  Lane i brings page i of the tile.
    const int shift = p.cache.page_shift;
    const int rows = shift >= 7 ? kTile : 1 << shift;    // rows of a box
    const int boxes = kTile / rows;                      // boxes of a tile and 64 channels
    int t = 0, s = 0;
    uint32_t ph = 0;
    bool ok = true, bad = false;
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 50);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int32_t* table = pc->table;
      const int t1 = pc->t1, end = pc->end, g = pc->g, outside = max(p.cache.n_pages, 1);   // (a page number the map does not have)
      auto page_of = [&](int tile) -> int {
        const int key = tile * kTile + lane * rows;
        if (lane >= boxes || tile >= t1 || key >= end) return outside;   // zeros
        const int pg = table[key >> shift];
        if ((unsigned)pg >= (unsigned)p.cache.n_pages) {
          bad = true;
          return outside;
        }
        return pg;
      };
      int page = page_of(pc->t0);
      for (int tile = pc->t0; tile < t1; ++tile) {
        const int slot = (tile * kTile + lane * rows) & ((1 << shift) - 1);
        const int next = page_of(tile + 1);
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->k_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 51)))) break;
        if (lane == 0) mbar_arrive_expect_tx(&sh->k_full[s], kTileBytes);
        __syncwarp();
        if (lane < boxes) {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_4d(smem_u32(k_smem + s * kTileBytes + h * kHalfBytes + lane * rows * 128), &tmap_k, h * 64, slot, g, page, &sh->k_full[s]);
        }
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->v_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 52)))) {
          mbar_wait_drain(&sh->k_full[s], ph, 20000ull);
          break;
        }
        if (lane == 0) mbar_arrive_expect_tx(&sh->v_full[s], kTileBytes);
        __syncwarp();
        if (lane < boxes) {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_4d(smem_u32(v_smem + s * kTileBytes + h * kHalfBytes + lane * rows * 128), &tmap_v, h * 64, slot, g, page, &sh->v_full[s]);
        }
        page = next;
        ++t;
        if (++s == kStages) { s = 0; ph ^= 1u; }
      }
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
    if (!ok) {
      // copies still landing in this CTA's shared memory get time to finish before it exits
      for (int back = 1; back <= kStages && back <= t; ++back) {
        const int u = t - back;
        mbar_wait_drain(&sh->k_full[u % kStages], (uint32_t)(u / kStages) & 1u, 20000ull);
        mbar_wait_drain(&sh->v_full[u % kStages], (uint32_t)(u / kStages) & 1u, 20000ull);
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer.  Per tile and block: the products of the tile before it (two steps of 64 keys), then the scores
    // of this one over the buffer those products read (the MMAs of one thread execute in the order they were issued).
    if (elect_one()) {
      const uint32_t idesc_s = make_idesc_bf16(kTile);
      // B operand with contiguous N (bit 16); fp16 operands have type number 0
      const uint32_t idesc_o = (kI8 ? (1u << 4) | ((uint32_t)(kD >> 3) << 17) | ((uint32_t)(128 >> 4) << 24) : make_idesc_bf16(kD)) | (1u << 16);
      bool ok = true;
      int t = 0;
      uint32_t kph = 0, vph = 0;
      int ks = 0, vs = 0;
      bool owed = false, owed_b = false, fresh = false;   // tile t - 1: products owed (of the second block too), first of its piece
      uint32_t cnt[2] = {0, 0};                           // tiles of a block whose products have been issued
      auto products = [&](int grp) -> bool {
        const uint64_t vdesc = desc_n_major(smem_u32(v_smem + vs * kTileBytes), kHalfBytes);
        const uint32_t p_tmem = tmem_base + (uint32_t)(grp * 128), o_tmem = tmem_base + kColO + (uint32_t)(grp * 128);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!mbar_wait(&sh->p_full[2 * grp + h], cnt[grp] & 1u, &sh->abort_flag, p.status, 55)) return false;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < 4; ++k)   // 16 keys: 2048 bytes of each channel block
            mma_bf16_ts(o_tmem, p_tmem + (uint32_t)(h * 64 + k * 8), vdesc + (uint64_t)((h * 64 + k * 16) * 128 >> 4), idesc_o,
                        (!fresh || h > 0 || k > 0) ? 1u : 0u);
          tc_commit(&sh->pv_done[2 * grp + h]);
        }
        ++cnt[grp];
        return true;
      };
      auto values_ready = [&]() -> bool {
        return mbar_wait(kI8 ? &sh->v_full[vs] : &sh->v_ok[vs], vph, &sh->abort_flag, p.status, 54);
      };
      auto values_done = [&]() {
        tc_commit(&sh->v_empty[vs]);
        if (++vs == kStages) { vs = 0; vph ^= 1u; }
      };
      int np = 0, nq[2] = {0, 0};
      for (;; ++np) {
        const Piece* pc = get_piece(np, ok, 53);
        if (!pc) break;
        const bool two = pc->n_rows > block_rows;
        const int t0 = pc->t0, t1 = pc->t1;
        for (int tile = t0; tile < t1 && ok; ++tile) {
          if (owed && !(ok = values_ready())) break;
          if (!(ok = mbar_wait(&sh->k_full[ks], kph, &sh->abort_flag, p.status, 57))) break;
          const uint64_t kdesc = make_b_desc(smem_u32(k_smem + ks * kTileBytes));
#pragma unroll 1
          for (int grp = 0; grp < 2 && ok; ++grp) {
            if (owed && (grp == 0 || owed_b) && !(ok = products(grp))) break;
            if (grp == 1 && !two) break;
            if (tile == t0) {
              if (!(ok = mbar_wait(&sh->q_full[grp], (uint32_t)nq[grp] & 1u, &sh->abort_flag, p.status, 58))) break;
              ++nq[grp];
            }
            tc_fence_after();
            const uint64_t qdesc = make_b_desc(smem_u32(q_smem + grp * kTileBytes));
#pragma unroll
            for (int k = 0; k < kD / 16; ++k) {
              const uint64_t off = (uint64_t)((k >> 2) * (kHalfBytes >> 4) + (k & 3) * 2);
              mma_bf16_ss(tmem_base + (uint32_t)(grp * 128), qdesc + off, kdesc + off, idesc_s, k ? 1u : 0u);
            }
            tc_commit(&sh->s_full[grp]);
            if (tile == t1 - 1) tc_commit(&sh->q_empty[grp]);
          }
          if (!ok) break;
          tc_commit(&sh->k_empty[ks]);
          if (++ks == kStages) { ks = 0; kph ^= 1u; }
          if (owed) values_done();
          owed = true;
          owed_b = two;
          fresh = tile == t0;
          ++t;
        }
        if (!ok) break;
      }
      if (ok && owed) {
        ok = values_ready() && products(0) && (!owed_b || products(1));
        if (ok) values_done();
      }
      if (!ok) {   // let every product already issued finish before tensor memory is freed
        tc_commit(&sh->drain);
        mbar_wait_drain(&sh->drain, 0, 2000000ull);
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---------------- walks the work line, publishes its pieces, and brings their queries
    const int64_t total = prefix[sc.b.n_seq];
    const int64_t share = sched_share(sc, total, gridDim.x);
    int64_t at = min(total, (int64_t)blockIdx.x * share);
    const int64_t stop = min(total, at + share);
    const int group = sc.group.d, block_tokens = block_rows / sc.group;
    KvRecord rec{};
    bool ok = true;
    int np = 0, nq[2] = {0, 0};
    while (ok) {
      Piece pc{};
      while (at < stop) {
        const KvUnit u = sched_unit<kMode>(sc, prefix, at, seqs);
        const int len = (int)min((int64_t)(u.tiles + sc.extra - u.skip), stop - at);
        pc.t0 = max(0, u.skip - sc.extra);
        pc.t1 = max(0, u.skip + len - sc.extra);
        const int64_t unit_at = at - u.skip;
        at += len;
        if (pc.t0 >= pc.t1) continue;
        pc.end = sched_end<kMode>(sc, u.s, u.rb);
        pc.ctx = kMode == kPrefix ? pc.end : u.s.n_all - u.s.n_new;
        pc.row0 = u.rb * sc.rows;
        pc.n_rows = min(sc.rows, u.s.n_new * group - pc.row0);
        pc.all_see = kMode == kPrefix || sc.b.perm ? pc.ctx : min(pc.end, pc.ctx + pc.row0 / sc.group + 1);
        pc.table = sc.b.page_table + (int64_t)u.b * sc.b.max_pages + (kMode == kOwn ? page0[u.b] : 0);
        pc.more = kMode == kOwn && page0[u.b] > 0;
        pc.g = u.g;
        pc.begin = u.s.begin;
        pc.whole = pc.t0 == 0 && pc.t1 == u.tiles;
        if (pc.t0 == 0 && !pc.whole) {
          pc.n_parts = (int)((unit_at + sc.extra + u.tiles - 1) / share) - (int)blockIdx.x + 1;
          rec.n_parts = pc.n_parts; rec.begin = pc.begin; rec.row0 = pc.row0; rec.n_rows = pc.n_rows; rec.g = pc.g;
        }
        break;
      }
      // (the other roles are done with a piece no later than the softmax warps, which have its last products)
      if (np >= kRing && !(ok = warp_all(mbar_wait(&sh->piece_empty[np % kRing], (uint32_t)(np / kRing - 1) & 1u, &sh->abort_flag, p.status, 64)))) break;
      if (lane == 0) {
        ring[np % kRing] = pc;
        mbar_arrive(&sh->piece_full[np % kRing]);
      }
      __syncwarp();
      if (pc.t0 >= pc.t1) break;
      const int blocks = pc.n_rows > block_rows ? 2 : 1;
      for (int k = 0; k < blocks; ++k) {
        if (nq[k] >= 1 && !(ok = warp_all(mbar_wait(&sh->q_empty[k], (uint32_t)(nq[k] - 1) & 1u, &sh->abort_flag, p.status, 56)))) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&sh->q_full[k], (uint32_t)(block_rows * 128 * kHalves));
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_3d(smem_u32(q_smem + k * kTileBytes + h * kHalfBytes), &tmap_q, h * 64, pc.g * group,
                        pc.begin + pc.row0 / sc.group + k * block_tokens, &sh->q_full[k]);
        }
        __syncwarp();
        ++nq[k];
      }
      ++np;
    }
    if (!ok)
      for (int k = 0; k < 2; ++k)
        if (nq[k]) mbar_wait_drain(&sh->q_full[k], (uint32_t)(nq[k] - 1) & 1u, 20000ull);
    if (kMode == kPlain && lane == 0) p.parts.rec[blockIdx.x] = rec;
  } else if (!kI8 && warp == 3) {
    // ---------------- looks through value tiles that not all rows see in full
    const int shift = p.cache.page_shift, rows = shift >= 7 ? kTile : 1 << shift;   // (of a box)
    int t = 0;
    bool ok = true;
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 60);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int t1 = pc->t1, end = pc->end, all_see = pc->all_see;
      bool poison = false;
      for (int tile = pc->t0; tile < t1; ++tile, ++t) {
        const int s = t % kStages;
        if (!(ok = warp_all(mbar_wait(&sh->v_full[s], (uint32_t)(t / kStages) & 1u, &sh->abort_flag, p.status, 60)))) break;
        if (tile * kTile + kTile > all_see) {
          uint8_t* vt = v_smem + s * kTileBytes;
          const int n_ok = end - tile * kTile;             // rows of the tile that hold keys
          bool wrote = false;
          // rows behind the last key: those of its own page hold anything (pages that were not asked for arrived as zeros)
          const int stale = min(kTile, (n_ok + rows - 1) & ~(rows - 1));
          if (n_ok < stale) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
              for (int c = n_ok * 8 + lane; c < stale * 8; c += 32) *reinterpret_cast<uint4*>(vt + h * kHalfBytes + c * 16) = make_uint4(0u, 0u, 0u, 0u);
            wrote = true;
          }
          bool hit = false;
          if (all_see < end) {
            __syncwarp();
            // the largest magnitude of the 16-bit halves shows an infinity or NaN (among the rows that not all see)
            uint32_t part[4] = {0u, 0u, 0u, 0u};
            const int first = max(0, all_see - tile * kTile) * 8;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              const uint4* vh = reinterpret_cast<const uint4*>(vt + h * kHalfBytes);
#pragma unroll 8
              for (int c = (first & ~31) + lane; c < kTile * 8; c += 32) {
                const uint4 v = vh[c];
                part[0] = __vmaxu2(part[0], v.x & 0x7fff7fffu);
                part[1] = __vmaxu2(part[1], v.y & 0x7fff7fffu);
                part[2] = __vmaxu2(part[2], v.z & 0x7fff7fffu);
                part[3] = __vmaxu2(part[3], v.w & 0x7fff7fffu);
              }
            }
            const uint32_t top = __vmaxu2(__vmaxu2(part[0], part[1]), __vmaxu2(part[2], part[3]));
            hit = __any_sync(0xffffffffu, (top & 0xffffu) >= 0x7f80u || (top >> 16) >= 0x7f80u);
          }
          if (hit) {
#pragma unroll 1
            for (int c = 0; c < kTileBytes / 512; ++c) {
              uint4* at16 = reinterpret_cast<uint4*>(vt + (c * 32 + lane) * 16);
              const uint4 v = *at16;
              uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
                if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu;
              }
              *at16 = make_uint4(w[0], w[1], w[2], w[3]);
            }
            wrote = true;
          }
          if (wrote) fence_proxy_async_smem();
          if (hit && !poison) {
            poison = true;
            if (lane == 0) *reinterpret_cast<volatile int*>(&ring[np % kRing].poison) = 1;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->v_ok[s]);
      }
    }
  } else if (warp >= 4 && warp < 12) {
    // ---------------- softmax warps: group grp = warps 4 + 4 grp .. works on block grp of every unit that has one
    const int quarter = warp & 3, grp = (warp - 4) >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_base = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_base = lane_base + (uint32_t)(grp * 128), o_addr = lane_base + kColO + (uint32_t)(grp * 128);
    int32_t* kp = kp_all + (warp - 4) * kTile;
    bool ok = true;
    uint32_t cnt = 0;                            // tiles of this group so far
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 62);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int unit_row = grp * block_rows + row;       // row of the unit
      if (grp * block_rows >= pc->n_rows) {              // (the second group of a unit of one block)
        if (lane == 0) mbar_arrive(&sh->piece_empty[np % kRing]);
        continue;
      }
      const bool live = row < block_rows && unit_row < pc->n_rows;
      const int ctx = pc->ctx, end = pc->end, t1 = pc->t1;
      const int32_t* perm = kMode != kPrefix && sc.b.perm ? sc.b.perm + pc->begin : nullptr;
      const int tok = live ? (pc->row0 + unit_row) / sc.group : 0;
      const int all_see = kMode == kPrefix ? end : perm ? ctx : min(end, ctx + (pc->row0 + grp * block_rows) / sc.group + 1);   // of this block
      // live rows: without perm, keys below lim; with it, the context and the chunk's rows whose index is at most lim
      const int lim = kMode == kPrefix ? (live ? end : 0) : perm ? (live ? perm[tok] : INT_MIN) : live ? min(end, ctx + tok + 1) : 0;
      // The maximum is found before the scale is applied, and a masked score is -inf times it: both want a positive scale. A head
      // whose static scale is not one (zero where every key was zero) has its scores scaled first.
      const float given = p.scale * 1.4426950408889634f * (kI8 ? p.cache.k_scale[pc->g] : 1.0f);
      const bool scale_first = kI8 && !(given >= FLT_MIN);
      const float scale_log2 = scale_first ? 1.0f : given;
      const float lag_raw = kLag / scale_log2, lift_raw = kI8 ? kLiftChunk / scale_log2 : 0.0f;
      float m_used = -1.0e30f, l_run = 0.0f;   // the exponents' reference (raw units), the sum relative to it
      bool begun = false;                      // the accumulator holds products of this piece
      // ranks of the keys of the next masked tile, asked for a tile ahead
      int32_t rank_next[4];
      auto ask_ranks = [&](int tile) {
        if (perm && tile < t1 && tile * kTile + kTile > all_see) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int j = tile * kTile + c * 32 + lane;
            rank_next[c] = j >= end ? INT_MAX : j < ctx ? -1 : perm[j - ctx];
          }
        }
      };
      ask_ranks(pc->t0);
      for (int tile = pc->t0; tile < t1 && ok; ++tile, ++cnt) {
        const bool masked = tile * kTile + kTile > all_see;           // (also where the tile passes `end`)
        if (masked && perm) {
          __syncwarp();
#pragma unroll
          for (int c = 0; c < 4; ++c) kp[c * 32 + lane] = rank_next[c];
          __syncwarp();
        }
        ask_ranks(tile + 1);
        if (!(ok = warp_all(mbar_wait(&sh->s_full[grp], cnt & 1u, &sh->abort_flag, p.status, 59)))) break;
        tc_fence_after();
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const uint32_t s_addr = s_base + (uint32_t)(h * 64);
          uint32_t sv[64];
          tmem_ld_x32(s_addr, *reinterpret_cast<uint32_t (*)[32]>(&sv[0]));
          tmem_ld_x32(s_addr + 32u, *reinterpret_cast<uint32_t (*)[32]>(&sv[32]));
          tmem_wait_ld();
          if (kI8 && scale_first) {
#pragma unroll
            for (int e = 0; e < 64; ++e) sv[e] = __float_as_uint(__uint_as_float(sv[e]) * given);
          }
          if (masked) {
            if (perm) {
#pragma unroll
              for (int e4 = 0; e4 < 64; e4 += 4) {
                const int4 k4 = *reinterpret_cast<const int4*>(kp + h * 64 + e4);
                if (k4.x > lim) sv[e4] = 0xff800000u;
                if (k4.y > lim) sv[e4 + 1] = 0xff800000u;
                if (k4.z > lim) sv[e4 + 2] = 0xff800000u;
                if (k4.w > lim) sv[e4 + 3] = 0xff800000u;
              }
            } else {
              const int n = lim - (tile * kTile + h * 64);   // visible ones among the 64
#pragma unroll
              for (int e = 0; e < 64; ++e)
                if (e >= n) sv[e] = 0xff800000u;
            }
          }
          float mx[4] = {-1.0e30f, -1.0e30f, -1.0e30f, -1.0e30f};
#pragma unroll
          for (int e = 0; e < 64; ++e) mx[e & 3] = fmaxf(mx[e & 3], __uint_as_float(sv[e]));
          const float m_new = fmaxf(m_used, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) - lift_raw);
          // (only rows with a result have a say: what stands in the others is the next sequence's tokens, or nothing)
          if (__any_sync(0xffffffffu, live && m_new > m_used + lag_raw)) {
            if (begun) {
              // every earlier product must have landed: for the first step the scores behind it say so (their MMAs were issued
              // after those products), for the second the first step's own product has to be waited for
              if (h == 1 && !(ok = warp_all(mbar_wait(&sh->pv_done[2 * grp], cnt & 1u, &sh->abort_flag, p.status, 61)))) break;
              tc_fence_after();
              const float f = kv_exp2((m_used - m_new) * scale_log2);
#pragma unroll
              for (int cb = 0; cb < kD; cb += 16) {
                uint32_t v[16];
                tmem_ld_x16(o_addr + (uint32_t)cb, v);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                tmem_st_x16(o_addr + (uint32_t)cb, v);
              }
              tmem_wait_st();
              l_run *= f;
            }
            m_used = m_new;
          }
          begun = true;
          const float2 scale2 = make_float2(scale_log2, scale_log2);
          const float bias = -m_used * scale_log2;
          const float2 bias2 = make_float2(bias, bias);
          float2 sum2[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
          uint32_t pk[32];
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(sv[e]), __uint_as_float(sv[e + 1])), scale2, bias2);
            const float2 pr = make_float2(kv_exp2(x.x), kv_exp2(x.y));
            sum2[(e >> 1) & 1] = __fadd2_rn(sum2[(e >> 1) & 1], pr);
            pk[e >> 1] = kI8 ? kv_pack_f16(pr.x, pr.y) : kv_pack_bf16(pr.x, pr.y);
          }
          tmem_st_x32(s_addr, pk);
          tmem_wait_st();
          l_run += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh->p_full[2 * grp + h]);
        }
      }
      // ---- end of the piece: the result, or the partial one
      if (ok) ok = warp_all(mbar_wait(&sh->pv_done[2 * grp + 1], (cnt - 1) & 1u, &sh->abort_flag, p.status, 63));
      if (!ok) break;
      tc_fence_after();
      const bool whole = pc->whole != 0, bf16_out = whole && kMode == kPlain;
      const float vsc = kI8 ? p.cache.v_scale[pc->g] : 1.0f;
      const float w = bf16_out ? (l_run != 0.0f ? vsc / l_run : 0.0f) : vsc;
      const int64_t at_part = (int64_t)(2 * (int)blockIdx.x + (pc->t0 == 0 ? 1 : 0)) * kPitch + unit_row;
      const int head = pc->g * sc.group.d + (pc->row0 + unit_row) - tok * sc.group.d;
      const int64_t out_row = (int64_t)(pc->begin + tok), at_row = out_row * p.out.n_q_heads + head;
      if (kMode != kPlain && live && pc->t0 == 0) p.whole.ref[at_row] = KvRowRef{(int)blockIdx.x, pc->n_parts, unit_row, pc->more};
      const bool poison = !kI8 && *reinterpret_cast<const volatile int*>(&pc->poison) != 0;
      // Four neighbouring lanes exchange 16-byte pieces so that they write 64 contiguous bytes of one row after the other (a
      // lane writing its own row makes every store instruction touch 32 lines: 10 instead of 4 k cycles per piece).
      const uint8_t* mine = bf16_out ? reinterpret_cast<const uint8_t*>(p.out.O + out_row * p.out.ldo + (int64_t)head * kD)
                            : reinterpret_cast<const uint8_t*>(whole ? p.whole.o + at_row * kD : p.parts.o + at_part * kD);
      uint8_t* dst[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        dst[k] = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, live ? reinterpret_cast<unsigned long long>(mine) : 0ull, (lane & ~3) | k));
#pragma unroll 1
      for (int cb = 0; cb < kD; cb += 32) {
        uint32_t a[32];
        tmem_ld_x32(o_addr + (uint32_t)cb, a);
        tmem_wait_ld();
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(a[e]) * w;
        if (poison && live) {
          // rare: add what was taken out, for the keys of those tiles that this row sees
          const int first = max(max(pc->t0 * kTile, pc->all_see / kTile * kTile), 0), last = min(end, t1 * kTile);
          for (int key = first; key < last; ++key) {
            const bool sees = key < ctx || (perm ? perm[key - ctx] <= lim : key < lim);
            if (!sees) continue;
            const int pg = pc->table[key >> p.cache.page_shift];
            if ((unsigned)pg >= (unsigned)p.cache.n_pages) continue;
            const uint16_t* vr = reinterpret_cast<const uint16_t*>(p.cache.V + (int64_t)pg * p.cache.page_stride + (int64_t)pc->g * p.cache.head_stride +
                                                                  (int64_t)(key & ((1 << p.cache.page_shift) - 1)) * p.cache.slot_stride) + cb;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const uint32_t bits = (uint32_t)vr[e] << 16;
              if ((bits & 0x7f800000u) == 0x7f800000u) o[e] += __uint_as_float(bits);
            }
          }
        }
        if (bf16_out) {
          uint4 v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[k] = make_uint4(kv_pack_bf16(o[8 * k], o[8 * k + 1]), kv_pack_bf16(o[8 * k + 2], o[8 * k + 3]), kv_pack_bf16(o[8 * k + 4], o[8 * k + 5]),
                              kv_pack_bf16(o[8 * k + 6], o[8 * k + 7]));
          quad_transpose(v, lane);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (dst[k]) *reinterpret_cast<uint4*>(dst[k] + cb * 2 + (lane & 3) * 16) = v[k];
        } else {
#pragma unroll
          for (int e = 0; e < 32; e += 16) {
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              v[k] = make_uint4(__float_as_uint(o[e + 4 * k]), __float_as_uint(o[e + 4 * k + 1]), __float_as_uint(o[e + 4 * k + 2]), __float_as_uint(o[e + 4 * k + 3]));
            quad_transpose(v, lane);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (dst[k]) *reinterpret_cast<uint4*>(dst[k] + (cb + e) * 4 + (lane & 3) * 16) = v[k];
          }
        }
      }
      if (live) {
        const float m = l_run != 0.0f ? m_used * scale_log2 : -INFINITY;
        if (!whole) p.parts.ml[at_part] = make_float2(m, l_run);
        else if (kMode != kPlain) p.whole.ml[at_row] = make_float2(m, l_run);
        else if (p.out.lse) p.out.lse[at_row] = l_run != 0.0f ? (m + log2f(l_run)) * 0.6931471805599453f : -INFINITY;
      }
      tc_fence_before();   // the accumulator has been read before the next piece's first product replaces it
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->piece_empty[np % kRing]);
    }
  } else if (kI8 && warp >= 12) {
    // ---------------- int8 cache: four warps widen the codes into the operand tiles.  A thread owns one key of the tile; the
    // codes of the next tile are on their way while this one waits for its slot.
    const int r = (warp - 12) * 32 + lane, shift = p.cache.page_shift;
    constexpr int kLoads = kD / 16;
    int t = 0, s = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int np = 0; ok; ++np) {
      const Piece* pc = get_piece(np, ok, 65);
      if (!(ok = warp_all(ok)) || !pc) break;
      const int32_t* table = pc->table;
      const int t1 = pc->t1, end = pc->end;
      const int64_t head_off = (int64_t)pc->g * p.cache.head_stride;
      auto row_of = [&](int tile) -> int64_t {   // byte offset of this thread's row, -1 where it reads as zeros
        const int key = tile * kTile + r;
        if (tile >= t1 || key >= end) return -1;
        const int pg = table[key >> shift];
        if ((unsigned)pg >= (unsigned)p.cache.n_pages) {
          atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
          return -1;
        }
        return (int64_t)pg * p.cache.page_stride + head_off + (int64_t)(key & ((1 << shift) - 1)) * p.cache.slot_stride;
      };
      auto load = [&](const uint8_t* pool, int64_t off, uint4 (&x)[kLoads]) {
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
          x[c] = make_uint4(0u, 0u, 0u, 0u);
          if (off >= 0) x[c] = *reinterpret_cast<const uint4*>(pool + off + c * 16);
        }
      };
      int64_t off = row_of(pc->t0), off_next;
      uint4 kx[kLoads], vx[kLoads];
      load(p.cache.K, off, kx);
      for (int tile = pc->t0; tile < t1; ++tile) {
        load(p.cache.V, off, vx);
        off_next = row_of(tile + 1);
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->k_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 66)))) break;
        uint8_t* kd = k_smem + s * kTileBytes + r * 128;
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {   // 16 codes: two pieces
          uint4 a, b;
          i8x4_to_bf16(kx[c].x, a.x, a.y); i8x4_to_bf16(kx[c].y, a.z, a.w);
          i8x4_to_bf16(kx[c].z, b.x, b.y); i8x4_to_bf16(kx[c].w, b.z, b.w);
          uint8_t* blk = kd + (c >> 2) * kHalfBytes;
          *reinterpret_cast<uint4*>(blk + ((((2 * c) & 7) ^ (r & 7)) << 4)) = a;
          *reinterpret_cast<uint4*>(blk + ((((2 * c + 1) & 7) ^ (r & 7)) << 4)) = b;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->k_full[s]);
        load(p.cache.K, off_next, kx);
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->v_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 67)))) break;
        uint8_t* vd = v_smem + s * kTileBytes + r * 128;
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
          uint4 a, b;
          i8x4_to_f16(vx[c].x, a.x, a.y); i8x4_to_f16(vx[c].y, a.z, a.w);
          i8x4_to_f16(vx[c].z, b.x, b.y); i8x4_to_f16(vx[c].w, b.z, b.w);
          uint8_t* blk = vd + (c >> 2) * kHalfBytes;
          *reinterpret_cast<uint4*>(blk + ((((2 * c) & 7) ^ (r & 7)) << 4)) = a;
          *reinterpret_cast<uint4*>(blk + ((((2 * c + 1) & 7) ^ (r & 7)) << 4)) = b;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->v_full[s]);
        off = off_next;
        ++t;
        if (++s == kStages) { s = 0; ph ^= 1u; }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
  kv_end<kMode>();
}

template <int kD, bool kI8, KvMode kMode>
int launch(const KvAttnArgs& a, int workers, cudaStream_t st) {
  using C = ChunkCfg<kD, kI8>;
  constexpr int kHeld = kMode == kPlain ? kSeqsHeld : kMaxSharedSeqs, kPerSeq = (int)sizeof(int64_t) + kSeqBytes<kMode>;
  constexpr int kMost = kMode != kPlain ? (kMaxSharedSeqs + 1) * kPerSeq
                        : (kMaxKvSeqs + 1) * 8 > (kSeqsHeld + 1) * kPerSeq ? (kMaxKvSeqs + 1) * 8 : (kSeqsHeld + 1) * kPerSeq;
  static_assert(C::kSmem + kMost <= 232448, "shared memory of one CTA");
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_chunk_kernel<kD, kI8, kMode>, C::kSmem + kMost)) return MQ_ERR_CUDA;
  CUtensorMap mq_{}, mk{}, mv{};
  if (!encode_queries(&mq_, a.Q, a.ldq, a.out.n_q_heads, a.sched.b.total_q, a.sched.group.d, a.sched.rows / 2, kD)) return MQ_ERR_CUDA;
  if (!kI8 && (!encode_pages(&mk, a.cache.K, a.Q, a.cache, kD, kTile) || !encode_pages(&mv, a.cache.V, a.Q, a.cache, kD, kTile))) return MQ_ERR_CUDA;
  const size_t seqs = (size_t)a.sched.b.n_seq + 1;
  const cudaError_t e = launch_pdl(kv_chunk_kernel<kD, kI8, kMode>, dim3((unsigned)workers), dim3(C::kThreads),
                                   C::kSmem + seqs * (a.sched.b.n_seq <= kHeld ? kPerSeq : sizeof(int64_t)), st, mq_, mk, mv, a);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}
template <int kD, bool kI8>
int launch(const KvAttnArgs& a, KvMode mode, int workers, cudaStream_t st) {
  return mode == kPlain ? launch<kD, kI8, kPlain>(a, workers, st)
         : mode == kPrefix ? launch<kD, kI8, kPrefix>(a, workers, st) : launch<kD, kI8, kOwn>(a, workers, st);
}

}  // namespace

// Rows of a unit for a group size: two blocks of whole tokens (0: a token's heads do not fit into a block).
void kv_chunk_shape(int group, int* rows, int* pitch, int* tile, int* extra) {
  *rows = 2 * (kBlock / group) * group;
  *pitch = kPitch;
  *tile = kTile;
  *extra = kExtraTiles;
}

int launch_kv_chunk(const KvAttnArgs& a, KvMode mode, int dim, bool i8, int workers, cudaStream_t st) {
  if (dim == 128) return i8 ? launch<128, true>(a, mode, workers, st) : launch<128, false>(a, mode, workers, st);
  return i8 ? launch<64, true>(a, mode, workers, st) : launch<64, false>(a, mode, workers, st);
}

}  // namespace mq
