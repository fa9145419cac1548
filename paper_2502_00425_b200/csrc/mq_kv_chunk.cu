// Attention of long chunks over a paged key/value cache on the tensor cores (tcgen05), for units of 128 query rows.
//
// The work line, units and partial results are those of mq_kv_sched.cuh; one persistent CTA per SM walks its range of the
// line.  A row of a unit is (token, query head of the group), so every key tile serves the whole group.
//   S = Q K^T (128 rows x 128 keys, bf16, float32 accumulators in tensor memory);  P = exp2(scale (S - ref));  O += P V
//   * K and V tiles (128 keys) come straight from the pages by TMA: one box per page and 64 channels, 128-byte swizzle,
//     the page number as the outermost coordinate; what lies behind the last key is asked for at a page number outside
//     the map and arrives as zeros.  V is the second product's B operand as it lies (channels contiguous), no transpose.
//   * An int8 cache is read by four more warps, which widen the codes exactly (K to bf16, V to fp16) into the same tiles.
//   * Two groups of four softmax warps share every key tile (keys 0 .. 63 and 64 .. 127).  Each group has two score buffers and
//     its own output accumulator in tensor memory and runs an online softmax of its own; a thread owns one row.  P replaces the
//     scores it was made from and never leaves tensor memory.  The two results are merged when the unit's range ends.
//   * Tiles are numbered through over all units of a worker, so the products of the next unit's first tile are under way while
//     the softmax warps still write out the last unit; two more warps bring the next unit's queries.
//   * The exponents' reference may lag a row's maximum by 2^8 before the accumulator is rescaled.
// Visibility: a tile some row of the unit may not see in full is masked bit by bit, all others take no mask.  A value that some
// rows may not see must not reach them even if it is infinite or NaN: in masked tiles such values are replaced by zero in
// shared memory before the product, and added at the end of the range to the rows that do see them.
// Every wait is bounded (mq_sm100.cuh); an expired one makes all roles leave and sets the status word.
#include <cuda.h>

#include "mq_kv_sched.cuh"
#include "mq_sm100.cuh"

namespace mq {
namespace {

constexpr int kM = 128;                 // query rows of a unit
constexpr int kTile = 128;              // keys of a tile
constexpr int kHalfBytes = 128 * 128;   // 128 rows x 64 bf16, swizzled
constexpr int kStages = 2;
constexpr int kExtraTiles = 2;          // what a unit costs besides its tiles, in tiles
constexpr uint32_t kColO = 256;         // tensor memory: scores at 128 g + 64 b, outputs at 256 + 128 g
constexpr float kLag = 8.0f;            // log2 of how far a row's maximum may outgrow the reference
// fp16 probabilities (int8 cache): the reference lies 6 below the maximum, so they run to 2^6, and to 2^14 with the lag
constexpr float kLiftChunk = 6.0f;

struct ChunkBarriers {
  uint64_t q_full[2], q_empty[2];
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t s_full[4], p_full[4], pv_done[4];   // [2 group + buffer]
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
};

template <int kD, bool kI8>
struct ChunkCfg {
  static constexpr int kHalves = kD / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kThreads = (kI8 ? 16 : 12) * 32;
  static constexpr int kXch = 2 * kM * 2 * 4;   // [group][row][m, l]
  static constexpr int kSmem = 1024 + (2 + 2 * kStages) * kTileBytes + (int)sizeof(ChunkBarriers) + kXch + 8 * 64 * 4 + 16 * 8;
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// B operand whose N (64 channels per block, 128-byte swizzle) is contiguous: blocks `block_bytes` apart, 8-key groups 1024 apart
__device__ __forceinline__ uint64_t desc_n_major(uint32_t addr, uint32_t block_bytes) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(block_bytes >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

// What a worker does next on the line.
struct Piece {
  KvUnit u;
  int t0, t1, end, ctx, row0, n_rows;
  int64_t unit_at;
};
__device__ __forceinline__ bool next_piece(const KvSchedArgs& sc, const int64_t* prefix, int64_t& at, int64_t stop, Piece& p) {
  while (at < stop) {
    p.u = sched_unit(sc, prefix, at);
    const int len = (int)min((int64_t)(p.u.tiles + sc.extra - p.u.skip), stop - at);
    p.t0 = max(0, p.u.skip - sc.extra);
    p.t1 = max(0, p.u.skip + len - sc.extra);
    p.unit_at = at - p.u.skip;
    at += len;
    if (p.t0 < p.t1) {
      p.end = sched_end(sc, p.u.s, p.u.rb);
      p.ctx = p.u.s.n_all - p.u.s.n_new;
      p.row0 = p.u.rb * kM;
      p.n_rows = min(kM, p.u.s.n_new * sc.group - p.row0);
      return true;
    }
  }
  return false;
}

template <int kD, bool kI8>
__global__ void __launch_bounds__(ChunkCfg<kD, kI8>::kThreads, 1)
kv_chunk_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                const __grid_constant__ KvAttnArgs p) {
  using C = ChunkCfg<kD, kI8>;
  constexpr int kTileBytes = C::kTileBytes, kHalves = C::kHalves;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_smem = smem;                              // two buffers
  uint8_t* k_smem = q_smem + 2 * kTileBytes;
  uint8_t* v_smem = k_smem + kStages * kTileBytes;
  ChunkBarriers* sh = reinterpret_cast<ChunkBarriers*>(v_smem + kStages * kTileBytes);
  float* xch = reinterpret_cast<float*>(sh + 1);
  int32_t* kp_all = reinterpret_cast<int32_t*>(xch + 2 * kM * 2);   // [8 warps][64]
  int64_t* red = reinterpret_cast<int64_t*>(kp_all + 8 * 64);
  int64_t* prefix = red + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    if (!kI8) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_k)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmap_v)) : "memory");
    }
    const uint32_t fills = kI8 ? 4 : 1;   // who fills a tile: one TMA thread, or four widening warps
    for (int i = 0; i < 2; ++i) { mbar_init(&sh->q_full[i], 2); mbar_init(&sh->q_empty[i], 1); }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh->k_full[i], fills); mbar_init(&sh->k_empty[i], 1);
      mbar_init(&sh->v_full[i], fills); mbar_init(&sh->v_empty[i], 1);
    }
    for (int i = 0; i < 4; ++i) { mbar_init(&sh->s_full[i], 1); mbar_init(&sh->p_full[i], 4); mbar_init(&sh->pv_done[i], 1); }
    mbar_init(&sh->drain, 1);
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    tmem_alloc(&sh->tmem_base, 512);
    tmem_relinquish();
  }
  pdl_launch_dependents();
  pdl_wait();
  const KvSchedArgs& sc = p.sched;
  tc_fence_before();
  sched_prefix<C::kThreads>(sc, prefix, red);   // (ends with __syncthreads)
  tc_fence_after();
  const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t*>(&sh->tmem_base);
  const int64_t total = prefix[sc.b.n_seq];
  const int64_t share = sched_share(sc, total, gridDim.x);
  int64_t at = min(total, (int64_t)blockIdx.x * share);
  const int64_t stop = min(total, at + share);
  Piece pc;

  if (!kI8 && warp == 0) {
    // ---------------- TMA producer.  Lane i brings page i of the tile.
    const int shift = p.cache.page_shift;
    const int rows = shift >= 7 ? kTile : 1 << shift;    // rows of a box
    const int boxes = kTile / rows;                      // boxes of a tile and 64 channels
    int t = 0, s = 0;
    uint32_t ph = 0;
    bool ok = true, bad = false;
    while (ok && next_piece(sc, prefix, at, stop, pc)) {
      const int32_t* table = sc.b.page_table + (int64_t)pc.u.b * sc.b.max_pages;
      auto page_of = [&](int tile) -> int {
        const int key = tile * kTile + lane * rows;
        if (lane >= boxes || tile >= pc.t1 || key >= pc.end) return p.cache.n_pages;   // outside the map: zeros
        const int pg = table[key >> shift];
        if ((unsigned)pg >= (unsigned)p.cache.n_pages) {
          bad = true;
          return p.cache.n_pages;
        }
        return pg;
      };
      int page = page_of(pc.t0);
      for (int tile = pc.t0; tile < pc.t1; ++tile) {
        const int slot = (tile * kTile + lane * rows) & ((1 << shift) - 1);
        const int next = page_of(tile + 1);
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->k_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 51)))) break;
        if (lane == 0) mbar_arrive_expect_tx(&sh->k_full[s], kTileBytes);
        __syncwarp();
        if (lane < boxes) {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_4d(smem_u32(k_smem + s * kTileBytes + h * kHalfBytes + lane * rows * 128), &tmap_k, h * 64, slot, pc.u.g, page, &sh->k_full[s]);
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
            tma_load_4d(smem_u32(v_smem + s * kTileBytes + h * kHalfBytes + lane * rows * 128), &tmap_v, h * 64, slot, pc.u.g, page, &sh->v_full[s]);
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
    // ---------------- MMA issuer: per tile the scores of both groups, then the products of the tile before it (whose
    // accumulators start anew with a piece).  Scores of tile t overwrite the buffer that the product of tile t - 2 read,
    // which was issued earlier by this same thread.
    if (elect_one()) {
      const uint32_t idesc_s = make_idesc_bf16(64);
      const uint32_t idesc_o = (kI8 ? (1u << 4) | ((uint32_t)(kD >> 3) << 17) | ((uint32_t)(128 >> 4) << 24) : make_idesc_bf16(kD)) | (1u << 16);
      bool ok = true;
      int t = 0, np = 0, ks = 0, vs = 0;
      uint32_t kph = 0, vph = 0;
      bool first = false;   // tile t - 1 is the first of its piece
      auto issue_pv = [&](int u) -> bool {
        const int b = u & 1;
        const uint32_t par = (uint32_t)(u >> 1) & 1u;
        if (!mbar_wait(&sh->v_full[vs], vph, &sh->abort_flag, p.status, 54)) return false;
        const uint64_t vdesc = desc_n_major(smem_u32(v_smem + vs * kTileBytes), kHalfBytes);
#pragma unroll
        for (int grp = 0; grp < 2; ++grp) {
          if (!mbar_wait(&sh->p_full[2 * grp + b], par, &sh->abort_flag, p.status, 55)) return false;
          tc_fence_after();
          const uint32_t p_tmem = tmem_base + (uint32_t)(grp * 128 + b * 64), o_tmem = tmem_base + kColO + (uint32_t)(grp * 128);
#pragma unroll
          for (int k = 0; k < 4; ++k)   // 16 keys of the group: 2048 bytes of each channel block
            mma_bf16_ts(o_tmem, p_tmem + (uint32_t)(k * 8), vdesc + (uint64_t)((grp * 64 + k * 16) * 128 >> 4), idesc_o, (!first || k > 0) ? 1u : 0u);
          tc_commit(&sh->pv_done[2 * grp + b]);
        }
        tc_commit(&sh->v_empty[vs]);
        if (++vs == kStages) { vs = 0; vph ^= 1u; }
        return true;
      };
      while (ok && next_piece(sc, prefix, at, stop, pc)) {
        const int qb = np & 1;
        if (!(ok = mbar_wait(&sh->q_full[qb], (uint32_t)(np >> 1) & 1u, &sh->abort_flag, p.status, 53))) break;
        const uint64_t qdesc = make_b_desc(smem_u32(q_smem + qb * kTileBytes));
        for (int tile = pc.t0; tile < pc.t1 && ok; ++tile) {
          const int b = t & 1;
          if (!(ok = mbar_wait(&sh->k_full[ks], kph, &sh->abort_flag, p.status, 57))) break;
          tc_fence_after();
          const uint64_t kdesc = make_b_desc(smem_u32(k_smem + ks * kTileBytes));
#pragma unroll
          for (int grp = 0; grp < 2; ++grp) {
#pragma unroll
            for (int k = 0; k < kD / 16; ++k) {
              const uint64_t off = (uint64_t)((k >> 2) * (kHalfBytes >> 4) + (k & 3) * 2);
              mma_bf16_ss(tmem_base + (uint32_t)(grp * 128 + b * 64), qdesc + off, kdesc + off + (uint64_t)(grp * (64 * 128 >> 4)), idesc_s, k ? 1u : 0u);
            }
            tc_commit(&sh->s_full[2 * grp + b]);
          }
          tc_commit(&sh->k_empty[ks]);
          if (++ks == kStages) { ks = 0; kph ^= 1u; }
          if (tile == pc.t1 - 1) tc_commit(&sh->q_empty[qb]);
          if (t >= 1 && !(ok = issue_pv(t - 1))) break;
          first = tile == pc.t0;
          ++t;
        }
        ++np;
      }
      if (ok && t >= 1) ok = issue_pv(t - 1);
      if (!ok) {   // let every product already issued finish before tensor memory is freed
        tc_commit(&sh->drain);
        mbar_wait_drain(&sh->drain, 0, 2000000ull);
      }
    }
    __syncwarp();
  } else if (warp == 2 || warp == 3) {
    // ---------------- queries: two rows per thread, a buffer ahead of the products
    int np = 0;
    bool ok = true;
    while (ok && next_piece(sc, prefix, at, stop, pc)) {
      const int qb = np & 1;
      if (np >= 2 && !(ok = warp_all(mbar_wait(&sh->q_empty[qb], ((uint32_t)(np >> 1) & 1u) ^ 1u, &sh->abort_flag, p.status, 58)))) break;
      uint8_t* dst = q_smem + qb * kTileBytes;
      // neighbouring lanes take neighbouring 16-byte pieces of a row
      constexpr int kPieces = kD / 8, kSteps = kM * kPieces / 64;
#pragma unroll 1
      for (int c0 = 0; c0 < kSteps; c0 += 8) {
        uint4 v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const int idx = (c0 + c) * 64 + (warp - 2) * 32 + lane, r = idx / kPieces, pcs = idx % kPieces, row = pc.row0 + r;
          v[c] = make_uint4(0u, 0u, 0u, 0u);
          if (r < pc.n_rows)
            v[c] = *reinterpret_cast<const uint4*>(p.Q + (int64_t)(pc.u.s.begin + row / sc.group) * p.ldq +
                                                   (int64_t)(pc.u.g * sc.group + row % sc.group) * (kD * 2) + pcs * 16);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const int idx = (c0 + c) * 64 + (warp - 2) * 32 + lane, r = idx / kPieces, pcs = idx % kPieces;
          *reinterpret_cast<uint4*>(dst + (pcs >> 3) * kHalfBytes + r * 128 + (((pcs & 7) ^ (r & 7)) << 4)) = v[c];
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->q_full[qb]);
      ++np;
    }
  } else if (warp >= 4 && warp < 12) {
    // ---------------- softmax warps: group grp = warps 4 + 4 grp .. takes keys 64 grp .. of every tile
    const int quarter = warp & 3, grp = (warp - 4) >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_base = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t o_addr = lane_base + kColO + (uint32_t)(grp * 128);
    int32_t* kp = kp_all + (warp - 4) * 64;
    KvRecord rec{0, 0, 0, 0};
    bool ok = true;
    int t = 0;
    while (ok && next_piece(sc, prefix, at, stop, pc)) {
      const int32_t* perm = sc.b.perm ? sc.b.perm + pc.u.s.begin : nullptr;
      const bool live = row < pc.n_rows;
      const int tok = live ? (pc.row0 + row) / sc.group : 0;
      const int all_see = perm ? pc.ctx : min(pc.end, pc.ctx + pc.row0 / sc.group + 1);
      // live rows: without perm, keys below lim; with it, the context and the chunk's rows whose index is at most lim
      const int lim = perm ? (live ? perm[tok] : INT_MIN) : live ? min(pc.end, pc.ctx + tok + 1) : 0;
      const float scale_log2 = p.scale * 1.4426950408889634f * (kI8 ? p.cache.k_scale[pc.u.g] : 1.0f);
      const float lag_raw = kLag / scale_log2, lift_raw = kI8 ? kLiftChunk / scale_log2 : 0.0f;
      float m_used = -1.0e30f, l_run = 0.0f;   // the exponents' reference (raw units), the sum relative to it
      bool poison = false;                     // values were taken out of masked tiles
      for (int tile = pc.t0; tile < pc.t1 && ok; ++tile, ++t) {
        const int b = t & 1, vs = t % kStages;
        const uint32_t par = (uint32_t)(t >> 1) & 1u;
        const int base = tile * kTile + grp * 64;                     // this group's keys
        const bool masked = tile * kTile + kTile > all_see;           // (also where the tile passes `end`)
        uint32_t allowed_lo = ~0u, allowed_hi = ~0u;
        if (masked) {
          if (!perm) {
            const int n = min(max(lim - base, 0), 64);                // visible ones among the 64 (a dead row: none)
            allowed_lo = n >= 32 ? ~0u : (1u << n) - 1u;
            allowed_hi = n >= 64 ? ~0u : n > 32 ? (1u << (n - 32)) - 1u : 0u;
          } else {
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int j = base + c * 32 + lane;
              kp[c * 32 + lane] = j >= pc.end ? INT_MAX : j < pc.ctx ? -1 : perm[j - pc.ctx];
            }
            __syncwarp();
            allowed_lo = allowed_hi = 0u;
#pragma unroll 8
            for (int e = 0; e < 32; ++e) allowed_lo |= (uint32_t)(kp[e] <= lim) << e;
#pragma unroll 8
            for (int e = 0; e < 32; ++e) allowed_hi |= (uint32_t)(kp[32 + e] <= lim) << e;
          }
          // ---- this group's 64 rows of the value tile: zeros behind the last key, and no infinity or NaN
          if (!(ok = warp_all(mbar_wait(&sh->v_full[vs], (uint32_t)(t / kStages) & 1u, &sh->abort_flag, p.status, 60)))) break;
          if (!kI8) {
            uint8_t* vt = v_smem + vs * kTileBytes + grp * 64 * 128;
            bool hit = false;
#pragma unroll 2
            for (int c = 0; c < kHalves * 4; ++c) {
              const int idx = c * 128 + row;              // 16-byte piece of 64 rows x 128 bytes, per channel block
              uint4* at16 = reinterpret_cast<uint4*>(vt + (idx >> 9) * kHalfBytes + (idx & 511) * 16);
              uint4 v = *at16;
              uint32_t* w = reinterpret_cast<uint32_t*>(&v);
              bool fix = false;
              const bool behind = base + ((idx & 511) >> 3) >= pc.end;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; fix = true; }
                if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; fix = true; }
              }
              hit |= fix && !behind;
              if (behind) { v = make_uint4(0u, 0u, 0u, 0u); fix = true; }
              if (fix) *at16 = v;
            }
            poison |= __any_sync(0xffffffffu, hit);
            fence_proxy_async_smem();
          }
        }
        if (!(ok = warp_all(mbar_wait(&sh->s_full[2 * grp + b], par, &sh->abort_flag, p.status, 59)))) break;
        tc_fence_after();
        const uint32_t s_addr = lane_base + (uint32_t)(grp * 128 + b * 64);
        uint32_t sv[64];
        tmem_ld_x32(s_addr, *reinterpret_cast<uint32_t (*)[32]>(&sv[0]));
        tmem_ld_x32(s_addr + 32u, *reinterpret_cast<uint32_t (*)[32]>(&sv[32]));
        tmem_wait_ld();
        float mx[4] = {-1.0e30f, -1.0e30f, -1.0e30f, -1.0e30f};
        if (masked) {
#pragma unroll
          for (int e = 0; e < 64; ++e) {
            if (!(((e < 32 ? allowed_lo : allowed_hi) >> (e & 31)) & 1u)) sv[e] = 0xff800000u;
            mx[e & 3] = fmaxf(mx[e & 3], __uint_as_float(sv[e]));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 64; ++e) mx[e & 3] = fmaxf(mx[e & 3], __uint_as_float(sv[e]));
        }
        const float m_new = fmaxf(m_used, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) - lift_raw);
        if (__any_sync(0xffffffffu, m_new > m_used + lag_raw)) {
          if (tile > pc.t0) {
            // the product of the previous tile (and with it every earlier one) must have landed
            if (!(ok = warp_all(mbar_wait(&sh->pv_done[2 * grp + ((t - 1) & 1)], (uint32_t)((t - 1) >> 1) & 1u, &sh->abort_flag, p.status, 61)))) break;
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
        {
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
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->p_full[2 * grp + b]);
      }
      // ---- end of the range in this unit: merge the groups, write the result or the partial one
      if (ok) ok = warp_all(mbar_wait(&sh->pv_done[2 * grp + ((t - 1) & 1)], (uint32_t)((t - 1) >> 1) & 1u, &sh->abort_flag, p.status, 62));
      float* x = xch;
      x[(grp * kM + row) * 2] = m_used * scale_log2;
      x[(grp * kM + row) * 2 + 1] = l_run;
      tc_fence_before();
      // (values taken out of one group's half concern the other group's columns too)
      const bool all_ok = !named_bar_or(1, 256, !ok);
      const bool any_poison = !kI8 && named_bar_or(1, 256, poison);
      tc_fence_after();
      if (all_ok) {
        const float m0 = x[row * 2], l0 = x[row * 2 + 1], m1 = x[(kM + row) * 2], l1 = x[(kM + row) * 2 + 1];
        const float m = fmaxf(m0, m1);
        const float f0 = l0 != 0.0f ? kv_exp2(m0 - m) : 0.0f, f1 = l1 != 0.0f ? kv_exp2(m1 - m) : 0.0f;
        const float l = l0 * f0 + l1 * f1;
        const bool whole = pc.t0 == 0 && pc.t1 == pc.u.tiles;
        const float vsc = kI8 ? p.cache.v_scale[pc.u.g] : 1.0f;
        const float w = whole ? (l != 0.0f ? vsc / l : 0.0f) : vsc;
        const float w0 = f0 * w, w1 = f1 * w;
        const int slot = 2 * (int)blockIdx.x + (pc.t0 == 0 ? 1 : 0);
        const int head = pc.u.g * sc.group + (pc.row0 + row) % sc.group;
        const int64_t out_row = (int64_t)(pc.u.s.begin + tok);
        constexpr int kCols = kD / 2;                  // this thread's channels: kCols * grp ..
        __nv_bfloat16* dst = p.out.O + out_row * p.out.ldo + (int64_t)head * kD + grp * kCols;
        float* part = p.parts.o + ((int64_t)slot * kM + row) * kD + grp * kCols;
#pragma unroll 1
        for (int cb = 0; cb < kCols; cb += 16) {
          uint32_t a0[16], a1[16];
          tmem_ld_x16(lane_base + kColO + (uint32_t)(grp * kCols + cb), a0);
          tmem_ld_x16(lane_base + kColO + 128u + (uint32_t)(grp * kCols + cb), a1);
          tmem_wait_ld();
          float o[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = fmaf(__uint_as_float(a1[e]), w1, __uint_as_float(a0[e]) * w0);
          if (any_poison && live) {
            // rare: add what was taken out, for the keys of the masked tiles that this row sees
            const int first = max(pc.t0 * kTile, all_see / kTile * kTile), last = min(pc.end, pc.t1 * kTile);
            for (int key = max(first, 0); key < last; ++key) {
              const bool sees = key < pc.ctx || (perm ? perm[key - pc.ctx] <= lim : key < lim);
              if (!sees) continue;
              const int pg = sc.b.page_table[(int64_t)pc.u.b * sc.b.max_pages + (key >> p.cache.page_shift)];
              if ((unsigned)pg >= (unsigned)p.cache.n_pages) continue;
              const uint16_t* vr = reinterpret_cast<const uint16_t*>(p.cache.V + (int64_t)pg * p.cache.page_stride +
                                                                    (int64_t)pc.u.g * p.cache.head_stride +
                                                                    (int64_t)(key & ((1 << p.cache.page_shift) - 1)) * p.cache.slot_stride) +
                                   grp * kCols + cb;
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const uint32_t bits = (uint32_t)vr[e] << 16;
                if ((bits & 0x7f800000u) == 0x7f800000u) o[e] += __uint_as_float(bits);
              }
            }
          }
          if (live) {
            if (whole) {
#pragma unroll
              for (int e = 0; e < 16; e += 8)
                *reinterpret_cast<uint4*>(dst + cb + e) = make_uint4(kv_pack_bf16(o[e], o[e + 1]), kv_pack_bf16(o[e + 2], o[e + 3]),
                                                                     kv_pack_bf16(o[e + 4], o[e + 5]), kv_pack_bf16(o[e + 6], o[e + 7]));
            } else {
#pragma unroll
              for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(part + cb + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            }
          }
        }
        if (grp == 0 && live) {
          const float ml = l != 0.0f ? m : -INFINITY;
          if (!whole) p.parts.ml[(int64_t)slot * kM + row] = make_float2(ml, l);
          else if (p.out.lse) p.out.lse[out_row * p.out.n_q_heads + head] = l != 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
        if (pc.t0 == 0 && !whole) {
          rec.n_parts = (int)((pc.unit_at + sc.extra + pc.u.tiles - 1) / share) - (int)blockIdx.x + 1;
          rec.b = pc.u.b; rec.g = pc.u.g; rec.rb = pc.u.rb;
        }
      } else {
        ok = false;
      }
      // both groups' accumulators and the exchange have been read before the next unit's products and results replace them
      tc_fence_before();
      named_bar_sync(1, 256);
    }
    if (warp == 4 && lane == 0) p.parts.rec[blockIdx.x] = ok ? rec : KvRecord{0, 0, 0, 0};
  } else if (kI8 && warp >= 12) {
    // ---------------- int8 cache: four warps widen the codes into the operand tiles.  A thread owns one key of the tile; the
    // codes of the next tile are on their way while this one waits for its slot.
    const int r = (warp - 12) * 32 + lane, shift = p.cache.page_shift;
    constexpr int kLoads = kD / 16;
    int t = 0, s = 0;
    uint32_t ph = 0;
    bool ok = true;
    while (ok && next_piece(sc, prefix, at, stop, pc)) {
      const int32_t* table = sc.b.page_table + (int64_t)pc.u.b * sc.b.max_pages;
      auto row_of = [&](int tile) -> int64_t {   // byte offset of this thread's row, -1 where it reads as zeros
        const int key = tile * kTile + r;
        if (tile >= pc.t1 || key >= pc.end) return -1;
        const int pg = table[key >> shift];
        if ((unsigned)pg >= (unsigned)p.cache.n_pages) {
          atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
          return -1;
        }
        return (int64_t)pg * p.cache.page_stride + (int64_t)pc.u.g * p.cache.head_stride + (int64_t)(key & ((1 << shift) - 1)) * p.cache.slot_stride;
      };
      auto load = [&](const uint8_t* pool, int64_t off, uint4 (&x)[kLoads]) {
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
          x[c] = make_uint4(0u, 0u, 0u, 0u);
          if (off >= 0) x[c] = *reinterpret_cast<const uint4*>(pool + off + c * 16);
        }
      };
      int64_t off = row_of(pc.t0), off_next;
      uint4 kx[kLoads], vx[kLoads];
      load(p.cache.K, off, kx);
      for (int tile = pc.t0; tile < pc.t1; ++tile) {
        load(p.cache.V, off, vx);
        off_next = row_of(tile + 1);
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->k_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 63)))) break;
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
        if (t >= kStages && !(ok = warp_all(mbar_wait(&sh->v_empty[s], ph ^ 1u, &sh->abort_flag, p.status, 64)))) break;
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
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The pages as a map [page][head][slot][channel], read in boxes of 64 channels x (a page's slots, at most 128)
bool encode_pages(CUtensorMap* map, const uint8_t* base, const KvView& c, int dim) {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  if (!fn) return false;
  const int page = 1 << c.page_shift;
  const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)page, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)c.slot_stride, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride};
  const cuuint32_t box[4] = {64, (cuuint32_t)(page < kTile ? page : kTile), 1, 1};
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<uint8_t*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kD, bool kI8>
int launch(const KvAttnArgs& a, int workers, cudaStream_t st) {
  using C = ChunkCfg<kD, kI8>;
  static_assert(C::kSmem + (kMaxKvSeqs + 1) * 8 <= 232448, "shared memory of one CTA");
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_chunk_kernel<kD, kI8>, C::kSmem + (kMaxKvSeqs + 1) * (int)sizeof(int64_t))) return MQ_ERR_CUDA;
  CUtensorMap mk{}, mv{};
  if (!kI8 && (!encode_pages(&mk, a.cache.K, a.cache, kD) || !encode_pages(&mv, a.cache.V, a.cache, kD))) return MQ_ERR_CUDA;
  const cudaError_t e = launch_pdl(kv_chunk_kernel<kD, kI8>, dim3((unsigned)workers), dim3(C::kThreads),
                                   C::kSmem + ((size_t)a.sched.b.n_seq + 1) * sizeof(int64_t), st, mk, mv, a);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace

void kv_chunk_shape(int* rows, int* tile, int* extra) { *rows = kM; *tile = kTile; *extra = kExtraTiles; }

int launch_kv_chunk(const KvAttnArgs& a, int dim, bool i8, int workers, cudaStream_t st) {
  if (dim == 128) return i8 ? launch<128, true>(a, workers, st) : launch<128, false>(a, workers, st);
  return i8 ? launch<64, true>(a, workers, st) : launch<64, false>(a, workers, st);
}

}  // namespace mq
