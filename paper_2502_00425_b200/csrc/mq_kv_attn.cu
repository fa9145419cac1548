// Attention of the new tokens of a ragged batch over a paged key/value cache.
//
//   O[i, h] = sum_j P[i, j] V[j, g],  P = softmax_j(scale * Q[i, h] . K[j, g]),  lse = log of the denominator
//
// The kernel of this file is the one for few query rows (decode steps): it is bound by reading K and V once.  A unit is
// 16 query rows (tokens x the query heads of one key/value head), so a key is read once for the whole group.
//   * A warp is on its own: it streams 16 keys at a time (K and V rows, 16-byte asynchronous copies straight from the
//     pages, two or more tiles in flight) into its own ring in shared memory and runs a complete online softmax over
//     them on mma.sync; there is no block-wide barrier until the four warps' results are joined at the end of a range.
//     Tensor-core throughput is no concern here: at the cache's rate an SM sees 16 keys in about 190 cycles.
//   * The exponents are taken relative to the running maximum, the accumulator is rescaled only when a row's maximum moved.
//   * An int8 cache is read as codes and widened in registers to fp16 exactly (the products' sums do not care in which
//     order the channels come, so a thread takes contiguous codes); the scales multiply the scores and the result.
//     Queries are scaled by a power of two per row so that fp16 holds them with all their bits.
#include "mq_kv_sched.cuh"

namespace mq {
namespace {

constexpr int kM = 16;            // query rows of a unit
constexpr int kWarps = 4;
constexpr int kTile = 16 * kWarps; // keys of a tile: 16 per warp
constexpr int kThreads = kWarps * 32;
constexpr int kCtasPerSm = 3;
constexpr int kExtra = 3;         // what a unit costs besides its tiles, in tiles
// fp16 probabilities reach down to 2^-24 only: with the reference 14 below the maximum they run up to 2^14 instead of 1, and
// what is lost below is 2^-39 of the largest one (a sum over them stays in float32 either way).
constexpr float kLiftF16 = 14.0f;

template <int kD, bool kI8>
struct Cfg {
  static constexpr int kRow = kD * (kI8 ? 1 : 2);        // bytes of a cached row
  static constexpr int kStage = 16 * kRow * 2;           // K and V of 16 keys
  static constexpr int kStages = kI8 ? 4 : (kD == 128 ? 2 : 4);
  static constexpr int kRing = kStage * kStages;
  static constexpr int kSmem = kWarps * kRing;
  static_assert(kSmem >= kWarps * kM * kD * 4, "the join of the warps reuses the rings");
};

// Offset of 16-byte piece c of row r in a tile: pieces are exchanged within 128-byte lines so that the eight rows that
// one load instruction touches lie in different banks.
template <int kRow>
__device__ __forceinline__ uint32_t piece(int r, int c) {
  const uint32_t off = (uint32_t)r * kRow + (uint32_t)c * 16u;
  const uint32_t key = kRow >= 128 ? (uint32_t)r & 7u : ((uint32_t)r >> 1) & 7u;
  return off ^ (key << 4);
}

template <int kD, bool kI8>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
kv_decode_kernel(const __grid_constant__ KvAttnArgs p) {
  using C = Cfg<kD, kI8>;
  constexpr int kRow = C::kRow, kPieces = kRow / 16, kSteps = kD / 16, kOut = kD / 8;
  constexpr float kLift = kI8 ? kLiftF16 : 0.0f;   // m0, m1: the exponents' reference, the running maximum less this
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float ml_s[kWarps][kM][2];
  __shared__ int64_t red[kWarps];
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + C::kSmem);
  pdl_launch_dependents();
  pdl_wait();
  const KvSchedArgs& sc = p.sched;
  sched_prefix<kThreads>(sc, prefix, red);
  const int64_t total = prefix[sc.b.n_seq];
  const int64_t share = sched_share(sc, total, gridDim.x);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, t4 = lane & 3;
  KvRecord rec{};
  int64_t at = min(total, (int64_t)blockIdx.x * share);
  const int64_t stop = min(total, at + share);
  const uint32_t ring = kv_smem_u32(smem) + (uint32_t)(warp * C::kRing);
  while (at < stop) {
    const KvUnit u = sched_unit(sc, prefix, at);
    const int len = (int)min((int64_t)(u.tiles + sc.extra - u.skip), stop - at);   // of this range on the line
    const int t0 = max(0, u.skip - sc.extra), t1 = max(0, u.skip + len - sc.extra);
    const int64_t unit_at = at - u.skip;
    at += len;
    if (t0 == t1) continue;   // the range ends before the unit's first tile
    const int end = sched_end(sc, u.s, u.rb), ctx = u.s.n_all - u.s.n_new;
    const int row0 = u.rb * kM, n_rows = min(kM, u.s.n_new * sc.group - row0);
    const int32_t* table = sc.b.page_table + (int64_t)u.b * sc.b.max_pages;
    const int64_t head_off = (int64_t)u.g * p.cache.head_stride;

    // ---- the warp's stream of tiles: tile t holds keys (t * kWarps + warp) * 16 ..
    const int n_my = t1 - t0;
    auto page_of = [&](int i) -> int {   // the page of the i-th tile of this range, -1 where it holds no visible key
      const int key0 = ((t0 + i) * kWarps + warp) * 16;
      return i < n_my && key0 < end ? table[key0 >> p.cache.page_shift] : -1;
    };
    auto issue = [&](int i, int page) {
      if (i < n_my) {
        const int key0 = ((t0 + i) * kWarps + warp) * 16;
        int n_ok = min(max(end - key0, 0), 16);
        if (n_ok > 0 && (unsigned)page >= (unsigned)p.cache.n_pages) {
          n_ok = 0;
          if (lane == 0) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
        }
        const int64_t off = n_ok > 0 ? (int64_t)page * p.cache.page_stride + head_off +
                                           (int64_t)(key0 & ((1 << p.cache.page_shift) - 1)) * p.cache.slot_stride
                                     : 0;
        const uint32_t dst = ring + (uint32_t)((i % C::kStages) * C::kStage);
        constexpr int kCopies = 16 * kPieces / 32;
#pragma unroll
        for (int c = 0; c < kCopies; ++c) {
          const int idx = c * 32 + lane, r = idx / kPieces, pc = idx % kPieces;
          const bool ok = r < n_ok;
          const int64_t src = ok ? off + (int64_t)r * p.cache.slot_stride + pc * 16 : 0;
          const uint32_t d = dst + piece<kRow>(r, pc);
          cp_async16(d, ok ? p.cache.K + src : p.Q, ok ? 16u : 0u);
          cp_async16(d + 16 * kRow, ok ? p.cache.V + src : p.Q, ok ? 16u : 0u);
        }
      }
      cp_async_commit();
    };
    int page_next = page_of(0);
#pragma unroll
    for (int i = 0; i < C::kStages - 1; ++i) {
      const int pg = page_next;
      page_next = page_of(i + 1);
      issue(i, pg);
    }

    // ---- query fragments (A operand): rows quad and quad + 8
    uint32_t qf[kSteps][4];
    float sc0, sc1;                 // scores -> log2 units, per row
    const bool ok0 = quad < n_rows, ok1 = quad + 8 < n_rows;
    const int i0 = (row0 + quad) / sc.group, i1 = (row0 + quad + 8) / sc.group;
    {
      const int h0 = u.g * sc.group + (row0 + quad) % sc.group, h1 = u.g * sc.group + (row0 + quad + 8) % sc.group;
      const uint8_t* q0 = p.Q + (int64_t)(u.s.begin + i0) * p.ldq + (int64_t)h0 * (kD * 2);
      const uint8_t* q1 = p.Q + (int64_t)(u.s.begin + i1) * p.ldq + (int64_t)h1 * (kD * 2);
      sc0 = sc1 = p.scale * 1.4426950408889634f;
      if (!kI8) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const int c = (k * 16 + 2 * t4) * 2;
          qf[k][0] = ok0 ? *reinterpret_cast<const uint32_t*>(q0 + c) : 0u;
          qf[k][1] = ok1 ? *reinterpret_cast<const uint32_t*>(q1 + c) : 0u;
          qf[k][2] = ok0 ? *reinterpret_cast<const uint32_t*>(q0 + c + 16) : 0u;
          qf[k][3] = ok1 ? *reinterpret_cast<const uint32_t*>(q1 + c + 16) : 0u;
        }
      } else {
        // channel order of the product: step k, position (2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9) is channel t4 * D/4 + 4 k + 0 .. 3
        uint2 w0[kSteps], w1[kSteps];
        float m0 = 0.0f, m1 = 0.0f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const int c = (t4 * (kD / 4) + 4 * k) * 2;
          w0[k] = ok0 ? *reinterpret_cast<const uint2*>(q0 + c) : make_uint2(0u, 0u);
          w1[k] = ok1 ? *reinterpret_cast<const uint2*>(q1 + c) : make_uint2(0u, 0u);
          m0 = fmaxf(m0, fmaxf(fmaxf(fabsf(kv_bf16_lo(w0[k].x)), fabsf(kv_bf16_hi(w0[k].x))),
                               fmaxf(fabsf(kv_bf16_lo(w0[k].y)), fabsf(kv_bf16_hi(w0[k].y)))));
          m1 = fmaxf(m1, fmaxf(fmaxf(fabsf(kv_bf16_lo(w1[k].x)), fabsf(kv_bf16_hi(w1[k].x))),
                               fmaxf(fabsf(kv_bf16_lo(w1[k].y)), fabsf(kv_bf16_hi(w1[k].y)))));
        }
        m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 1)); m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 2));
        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 1)); m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 2));
        // the power of two that brings the row's largest magnitude into [1, 2) (an infinity stays one either way)
        const int e0 = m0 > 0.0f && m0 < INFINITY ? (int)((__float_as_uint(m0) >> 23) & 255) - 127 : 0;
        const int e1 = m1 > 0.0f && m1 < INFINITY ? (int)((__float_as_uint(m1) >> 23) & 255) - 127 : 0;
        const float f0 = exp2f((float)-e0), f1 = exp2f((float)-e1);
        const float ks = p.cache.k_scale[u.g];
        sc0 = sc0 * ks * exp2f((float)e0);
        sc1 = sc1 * ks * exp2f((float)e1);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          qf[k][0] = kv_pack_f16(kv_bf16_lo(w0[k].x) * f0, kv_bf16_hi(w0[k].x) * f0);
          qf[k][2] = kv_pack_f16(kv_bf16_lo(w0[k].y) * f0, kv_bf16_hi(w0[k].y) * f0);
          qf[k][1] = kv_pack_f16(kv_bf16_lo(w1[k].x) * f1, kv_bf16_hi(w1[k].x) * f1);
          qf[k][3] = kv_pack_f16(kv_bf16_lo(w1[k].y) * f1, kv_bf16_hi(w1[k].y) * f1);
        }
      }
    }
    // visibility: without perm, keys below lim; with it, the context and the chunk's rows whose index is not larger
    const int32_t* perm = sc.b.perm ? sc.b.perm + u.s.begin : nullptr;
    const int r_first = row0 / sc.group;
    const int all_see = perm ? ctx : min(end, ctx + r_first + 1);   // every row of the unit sees the keys below
    const int lim0 = ok0 ? (perm ? perm[i0] : ctx + i0 + 1) : INT_MIN, lim1 = ok1 ? (perm ? perm[i1] : ctx + i1 + 1) : INT_MIN;
    auto sees = [&](int key, int lim, bool ok) -> bool {
      if (key >= end || !ok) return false;
      if (!perm) return key < lim;
      return key < ctx || perm[key - ctx] <= lim;
    };

    float o[kOut][4];
#pragma unroll
    for (int n = 0; n < kOut; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;

    for (int i = 0; i < n_my; ++i) {
      const int pg = page_next;
      page_next = page_of(i + C::kStages);
      issue(i + C::kStages - 1, pg);
      cp_async_wait<C::kStages - 1>();
      __syncwarp();
      const uint32_t kt = ring + (uint32_t)((i % C::kStages) * C::kStage), vt = kt + 16 * kRow;
      const int key0 = ((t0 + i) * kWarps + warp) * 16;
      if (key0 < end) {
        float s[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
        if (!kI8) {
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            uint32_t b[4];
            ldsm_x4(kt + piece<kRow>((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), b);
            mma_16816<false>(s[0], qf[k], b[0], b[1]);
            mma_16816<false>(s[1], qf[k], b[2], b[3]);
          }
        } else {
          constexpr int kLoads = kD / 64;   // 16-byte loads per key row and thread
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int c = 0; c < kLoads; ++c) {
              uint32_t x[4];
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(kt + piece<kRow>(quad + 8 * j, t4 * kLoads + c)));
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                uint32_t b0, b1;
                i8x4_to_f16(x[w], b0, b1);
                mma_16816<true>(s[j], qf[4 * c + w], b0, b1);
              }
            }
          }
        }
        const bool masked = key0 + 16 > all_see;
        unsigned seen = 0xffu;   // bit 4 j + e: score s[j][e] counts
        if (masked) {
          seen = 0u;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (sees(key0 + 8 * j + 2 * t4 + (e & 1), e < 2 ? lim0 : lim1, e < 2 ? ok0 : ok1)) seen |= 1u << (4 * j + e);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[j][e] *= e < 2 ? sc0 : sc1;
            if (masked && !((seen >> (4 * j + e)) & 1u)) s[j][e] = -INFINITY;
          }
        float x0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), x1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1)); x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1)); x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
        x0 -= kLift;
        x1 -= kLift;
        if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1)) {
          const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
          const float f0 = m0 == -INFINITY ? 0.0f : kv_exp2(m0 - n0), f1 = m1 == -INFINITY ? 0.0f : kv_exp2(m1 - n1);
          m0 = n0; m1 = n1;
          l0 *= f0; l1 *= f1;
#pragma unroll
          for (int n = 0; n < kOut; ++n) { o[n][0] *= f0; o[n][1] *= f0; o[n][2] *= f1; o[n][3] *= f1; }
        }
        const float u0 = m0 == -INFINITY ? 0.0f : m0, u1 = m1 == -INFINITY ? 0.0f : m1;   // a row without keys yet: exp2(-inf) = 0
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          s[j][0] = kv_exp2(s[j][0] - u0); s[j][1] = kv_exp2(s[j][1] - u0);
          s[j][2] = kv_exp2(s[j][2] - u1); s[j][3] = kv_exp2(s[j][3] - u1);
          l0 += s[j][0] + s[j][1];
          l1 += s[j][2] + s[j][3];
        }
        // A value that some rows may not see must not reach them even if it is infinite or NaN (0 * inf): such a tile
        // is multiplied key by key.  Only tiles with rows of different sight can hold one.
        bool odd = false;
        if (!kI8 && masked && all_see < end) {
          bool mine = false;
#pragma unroll
          for (int c = 0; c < 16 * kPieces / 32; ++c) {
            uint32_t x[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(vt + (uint32_t)(c * 32 + lane) * 16u));
#pragma unroll
            for (int w = 0; w < 4; ++w) mine |= (x[w] & 0x7f80u) == 0x7f80u || (x[w] & 0x7f800000u) == 0x7f800000u;
          }
          odd = __any_sync(0xffffffffu, mine);
        }
        if (!kI8 && odd) {
#pragma unroll
          for (int key = 0; key < 16; ++key) {
            const int from = (lane & ~3) | ((key & 7) >> 1);
            const float p0 = __shfl_sync(0xffffffffu, s[key >> 3][key & 1], from), p1 = __shfl_sync(0xffffffffu, s[key >> 3][2 + (key & 1)], from);
            const unsigned vis = __shfl_sync(0xffffffffu, seen, from);
            const bool v0 = (vis >> (4 * (key >> 3) + (key & 1))) & 1u, v1 = (vis >> (4 * (key >> 3) + 2 + (key & 1))) & 1u;
#pragma unroll
            for (int n = 0; n < kOut; ++n) {
              uint32_t x;
              asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(vt + piece<kRow>(key, n) + (uint32_t)t4 * 4u));
              if (v0) { o[n][0] = fmaf(p0, kv_bf16_lo(x), o[n][0]); o[n][1] = fmaf(p0, kv_bf16_hi(x), o[n][1]); }
              if (v1) { o[n][2] = fmaf(p1, kv_bf16_lo(x), o[n][2]); o[n][3] = fmaf(p1, kv_bf16_hi(x), o[n][3]); }
            }
          }
        } else if (!kI8) {
          const uint32_t pf[4] = {kv_pack_bf16(s[0][0], s[0][1]), kv_pack_bf16(s[0][2], s[0][3]), kv_pack_bf16(s[1][0], s[1][1]),
                                  kv_pack_bf16(s[1][2], s[1][3])};
#pragma unroll
          for (int n = 0; n < kOut; n += 2) {
            uint32_t b[4];
            ldsm_x4_trans(vt + piece<kRow>((lane & 7) + (((lane >> 3) & 1) << 3), n + (lane >> 4)), b);
            mma_16816<false>(o[n], pf, b[0], b[1]);
            mma_16816<false>(o[n + 1], pf, b[2], b[3]);
          }
        } else {
          const uint32_t pf[4] = {kv_pack_f16(s[0][0], s[0][1]), kv_pack_f16(s[0][2], s[0][3]), kv_pack_f16(s[1][0], s[1][1]),
                                  kv_pack_f16(s[1][2], s[1][3])};
          // output column n of product j is channel n * D/8 + j: a thread reads D/8 contiguous codes of each of its four keys
          constexpr int kWords = kD / 32;
          uint32_t x[4][kWords];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = 2 * t4 + (r & 1) + 8 * (r >> 1);
            if (kD == 128)
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(x[r][0]), "=r"(x[r][1]), "=r"(x[r][2 % kWords]), "=r"(x[r][3 % kWords]) : "r"(vt + piece<kRow>(key, quad)));
            else
              asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];"
                           : "=r"(x[r][0]), "=r"(x[r][1]) : "r"(vt + piece<kRow>(key, quad >> 1) + (uint32_t)(quad & 1) * 8u));
          }
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            const uint32_t lo01 = __byte_perm(x[0][w], x[1][w], 0x5140), hi01 = __byte_perm(x[0][w], x[1][w], 0x7362);
            const uint32_t lo23 = __byte_perm(x[2][w], x[3][w], 0x5140), hi23 = __byte_perm(x[2][w], x[3][w], 0x7362);
            uint32_t a0, a1, b0, b1;
            i8x4_to_f16(lo01, a0, a1);
            i8x4_to_f16(lo23, b0, b1);
            mma_16816<true>(o[4 * w], pf, a0, b0);
            mma_16816<true>(o[4 * w + 1], pf, a1, b1);
            i8x4_to_f16(hi01, a0, a1);
            i8x4_to_f16(hi23, b0, b1);
            mma_16816<true>(o[4 * w + 2], pf, a0, b0);
            mma_16816<true>(o[4 * w + 3], pf, a1, b1);
          }
        }
      }
      __syncwarp();   // every lane has read the tile before its slot is filled again
    }
    cp_async_wait<0>();
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1); l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1); l1 += __shfl_xor_sync(0xffffffffu, l1, 2);

    // ---- join the warps: each ran a softmax over its own keys
    __syncthreads();   // the rings are free
    float* join = reinterpret_cast<float*>(smem) + warp * (kM * kD);
    if (t4 == 0) {
      ml_s[warp][quad][0] = m0; ml_s[warp][quad][1] = l0;
      ml_s[warp][quad + 8][0] = m1; ml_s[warp][quad + 8][1] = l1;
    }
#pragma unroll
    for (int n = 0; n < kOut; ++n) {
      if (!kI8) {
        *reinterpret_cast<float2*>(join + quad * kD + 8 * n + 2 * t4) = make_float2(o[n][0], o[n][1]);
        *reinterpret_cast<float2*>(join + (quad + 8) * kD + 8 * n + 2 * t4) = make_float2(o[n][2], o[n][3]);
      } else {
        join[quad * kD + (2 * t4) * kOut + n] = o[n][0];
        join[quad * kD + (2 * t4 + 1) * kOut + n] = o[n][1];
        join[(quad + 8) * kD + (2 * t4) * kOut + n] = o[n][2];
        join[(quad + 8) * kD + (2 * t4 + 1) * kOut + n] = o[n][3];
      }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == u.tiles;
    const int slot = 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0);
    const float vs = kI8 ? p.cache.v_scale[u.g] : 1.0f;
    constexpr int kColThreads = kD / 2;                 // two channels per thread
    const int col = ((int)threadIdx.x % kColThreads) * 2;
    for (int r = (int)threadIdx.x / kColThreads; r < n_rows; r += kThreads / kColThreads) {
      float m = ml_s[0][r][0];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) m = fmaxf(m, ml_s[w][r][0]);
      float l = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float mw = ml_s[w][r][0];
        const float f = mw == -INFINITY ? 0.0f : kv_exp2(mw - m);
        l = fmaf(f, ml_s[w][r][1], l);
        const float2 v = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(smem) + w * (kM * kD) + r * kD + col);
        if (f != 0.0f) { x = fmaf(f, v.x, x); y = fmaf(f, v.y, y); }
      }
      if (whole) {
        const int tok = u.s.begin + (row0 + r) / sc.group, head = u.g * sc.group + (row0 + r) % sc.group;
        const float inv = l == 0.0f ? 0.0f : vs / l;
        *reinterpret_cast<__nv_bfloat162*>(p.out.O + (int64_t)tok * p.out.ldo + (int64_t)head * kD + col) =
            __floats2bfloat162_rn(x * inv, y * inv);
        if (col == 0 && p.out.lse)
          p.out.lse[(int64_t)tok * p.out.n_q_heads + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      } else {
        if (col == 0) p.parts.ml[(int64_t)slot * kM + r] = make_float2(m, l);
        *reinterpret_cast<float2*>(p.parts.o + ((int64_t)slot * kM + r) * kD + col) = make_float2(x * vs, y * vs);
      }
    }
    if (t0 == 0 && !whole) {
      // the pieces end with the worker whose range holds the unit's last tile
      rec.n_parts = (int)((unit_at + sc.extra + u.tiles - 1) / share) - (int)blockIdx.x + 1;
      rec.begin = u.s.begin; rec.row0 = row0; rec.n_rows = n_rows; rec.g = u.g;
    }
    __syncthreads();   // the join has been read before the next range fills the rings
  }
  if (threadIdx.x == 0) p.parts.rec[blockIdx.x] = rec;
}

// Joins the pieces of the units that are split.  kWarps warps share a row and take every kWarps-th piece: four where
// a unit has few rows and may have tens of pieces (a decode step of one sequence is as long as this chain of loads),
// one where it has 128 rows and mostly two pieces.  The record holds all that is needed: one dependent load before
// the pieces.
constexpr int kJoinThreads = 256;
template <int kD, int kWarpsPerRow>
__global__ void __launch_bounds__(kJoinThreads)
kv_combine_kernel(const int pitch, const int group, const KvParts parts, const KvOutArgs out) {
  constexpr int kPer = kD / 32, kRows = kJoinThreads / 32 / kWarpsPerRow;
  __shared__ float part[kRows][kWarpsPerRow][kD + 2];
  pdl_launch_dependents();
  pdl_wait();
  const int w = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rr = warp / kWarpsPerRow, pw = warp % kWarpsPerRow;
  const KvRecord rec = parts.rec[w];
  if ((int)blockIdx.y * kRows >= (rec.n_parts ? rec.n_rows : 0)) return;
  const int r = blockIdx.y * kRows + rr;
  const bool live = r < rec.n_rows;
  auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * w + 1 : 2 * (w + i)) * pitch + r; };
  float m = -INFINITY, l = 0.0f, x[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
  if (live) {
    constexpr int kBatch = kWarpsPerRow > 1 ? 8 : 3;
    for (int i0 = pw; i0 < rec.n_parts; i0 += kBatch * kWarpsPerRow) {
      float2 ml[kBatch];
      float v[kBatch][kPer];
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        const int i = i0 + c * kWarpsPerRow;
        ml[c] = make_float2(-INFINITY, 0.0f);
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[c][e] = 0.0f;
        if (i < rec.n_parts) {
          const int64_t at = slot(i);
          ml[c] = parts.ml[at];
          const float* src = parts.o + at * kD + lane * kPer;
          if (kPer == 4) {
            const float4 q = *reinterpret_cast<const float4*>(src);
            v[c][0] = q.x; v[c][1] = q.y; v[c][2 % kPer] = q.z; v[c][3 % kPer] = q.w;
          } else {
            const float2 q = *reinterpret_cast<const float2*>(src);
            v[c][0] = q.x; v[c][1] = q.y;
          }
        }
      }
      float top = m;
#pragma unroll
      for (int c = 0; c < kBatch; ++c) top = fmaxf(top, ml[c].x);
      if (top == -INFINITY) continue;
      const float back = kv_exp2(m - top);   // (0 while nothing has been seen)
      l *= back;
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] *= back;
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        if (ml[c].x == -INFINITY) continue;
        const float f = kv_exp2(ml[c].x - top);
        l = fmaf(f, ml[c].y, l);
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = fmaf(f, v[c][e], x[e]);
      }
      m = top;
    }
  }
  if (kWarpsPerRow > 1) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) part[rr][pw][lane * kPer + e] = x[e];
    if (lane == 0) {
      part[rr][pw][kD] = m;
      part[rr][pw][kD + 1] = l;
    }
    __syncthreads();
    if (pw != 0) return;
    m = part[rr][0][kD];
#pragma unroll
    for (int k = 1; k < kWarpsPerRow; ++k) m = fmaxf(m, part[rr][k][kD]);
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < kWarpsPerRow; ++k) {
      const float mk = part[rr][k][kD];
      if (mk == -INFINITY) continue;
      const float f = kv_exp2(mk - m);
      l = fmaf(f, part[rr][k][kD + 1], l);
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] = fmaf(f, part[rr][k][lane * kPer + e], x[e]);
    }
  }
  if (!live) return;
  const int tok = rec.begin + (rec.row0 + r) / group, head = rec.g * group + (rec.row0 + r) % group;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  __nv_bfloat16* dst = out.O + (int64_t)tok * out.ldo + (int64_t)head * kD + lane * kPer;
  if (kPer == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(kv_pack_bf16(x[0] * inv, x[1] * inv), kv_pack_bf16(x[2 % kPer] * inv, x[3 % kPer] * inv));
  else
    *reinterpret_cast<uint32_t*>(dst) = kv_pack_bf16(x[0] * inv, x[1] * inv);
  if (lane == 0 && out.lse)
    out.lse[(int64_t)tok * out.n_q_heads + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <int kD, bool kI8>
int launch_decode(const KvAttnArgs& a, int workers, cudaStream_t st) {
  using C = Cfg<kD, kI8>;
  const size_t smem = C::kSmem + ((size_t)a.sched.b.n_seq + 1) * sizeof(int64_t);
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_decode_kernel<kD, kI8>, C::kSmem + (kMaxKvSeqs + 1) * (int)sizeof(int64_t))) return MQ_ERR_CUDA;
  const cudaError_t e = launch_pdl(kv_decode_kernel<kD, kI8>, dim3((unsigned)workers), dim3(kThreads), smem, st, a);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

// Which kernel, and how many workers.  Up to kFewRows query rows per key/value head (tokens x heads of the group) take the
// kernel above in blocks of 16 rows, more take the 128-row tensor-memory kernel of mq_kv_chunk.cu.
constexpr int kFewRows = 32;
struct Plan {
  bool chunk;
  int workers, rows, pitch, tile, extra;
};
Plan attn_plan(const mq_kv_batch* b, const mq_kv_cache* c, int group) {
  Plan p{};
  // (a token's heads have to fit into a block of that kernel, and its maps need a page)
  p.chunk = (int64_t)b->max_q * group > kFewRows && group <= 128 && c->n_pages > 0;
  if (p.chunk) kv_chunk_shape(group, &p.rows, &p.pitch, &p.tile, &p.extra);
  else p.rows = p.pitch = kM, p.tile = kTile, p.extra = kExtra;
  const int64_t blocks = ((int64_t)b->max_q * group + p.rows - 1) / p.rows;
  const int64_t tiles = (((int64_t)b->max_pages * c->page_size) + p.tile - 1) / p.tile;
  const int64_t most = (int64_t)b->n_seq * c->n_kv_heads * blocks * (tiles > 0 ? tiles : 1);
  const int64_t cap = (int64_t)sm_count() * (p.chunk ? 1 : kCtasPerSm);
  p.workers = (int)(most < cap ? (most > 0 ? most : 1) : cap);
  return p;
}

int check_attention(const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads, KvBatchView* bv, KvView* cv) {
  int rc = check_kv_cache(cache, cv);
  if (rc != MQ_OK) return rc;
  if ((rc = check_kv_batch(batch, bv)) != MQ_OK) return rc;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads) return MQ_ERR_INVALID_ARG;
  // row indices (token x head of the group) are int32
  if ((int64_t)batch->max_q * (n_q_heads / cache->n_kv_heads) > (1 << 30)) return MQ_ERR_UNSUPPORTED;
  return MQ_OK;
}

}  // namespace

namespace {
template <int kD, int kW>
cudaError_t launch_join(const KvSchedArgs& a, const KvParts& parts, const KvOutArgs& out, int workers, cudaStream_t st) {
  return launch_pdl(kv_combine_kernel<kD, kW>, dim3((unsigned)workers, (unsigned)(a.pitch * kW * 32 / kJoinThreads)), dim3(kJoinThreads), 0, st,
                    a.pitch, a.group, parts, out);
}
}  // namespace

int launch_kv_combine(const KvSchedArgs& a, const KvParts& parts, const KvOutArgs& out, int workers, int dim, cudaStream_t st) {
  const bool few = a.pitch == kM;
  const cudaError_t e = dim == 128 ? (few ? launch_join<128, 4>(a, parts, out, workers, st) : launch_join<128, 1>(a, parts, out, workers, st))
                                   : (few ? launch_join<64, 4>(a, parts, out, workers, st) : launch_join<64, 1>(a, parts, out, workers, st));
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_kv_attention_workspace_bytes(const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads) {
  KvBatchView bv;
  KvView cv;
  if (check_attention(batch, cache, n_q_heads, &bv, &cv) != MQ_OK) return 0;
  const Plan p = attn_plan(batch, cache, n_q_heads / cache->n_kv_heads);
  return kStatusBytes + kv_parts_bytes(p.workers, p.pitch, cache->head_dim);
}

extern "C" int mq_kv_attention(const void* Q, int64_t ldq, const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads,
                               float scale, void* O, int64_t ldo, float* lse, void* ws, size_t ws_bytes, void* stream) {
  KvAttnArgs a{};
  const int rc = check_attention(batch, cache, n_q_heads, &a.sched.b, &a.cache);
  if (rc != MQ_OK) return rc;
  if (!(scale > 0.0f) || !std::isfinite(scale)) return MQ_ERR_INVALID_ARG;
  const int64_t width = (int64_t)n_q_heads * cache->head_dim;
  if (ldq < width || ldo < width) return MQ_ERR_INVALID_ARG;
  if (batch->n_seq == 0 || batch->total_q == 0 || batch->max_q == 0) return MQ_OK;
  if (!Q || !O || !ws) return MQ_ERR_INVALID_ARG;
  if (!kv_aligned16(Q) || !kv_aligned16(O) || ldq % 8 || ldo % 8 || (reinterpret_cast<uintptr_t>(ws) & 255u)) return MQ_ERR_ALIGNMENT;
  const Plan p = attn_plan(batch, cache, n_q_heads / cache->n_kv_heads);
  if (ws_bytes < kStatusBytes + kv_parts_bytes(p.workers, p.pitch, cache->head_dim)) return MQ_ERR_WORKSPACE;
  a.Q = static_cast<const uint8_t*>(Q);
  a.ldq = ldq * 2;
  a.sched.page_shift = a.cache.page_shift;
  a.sched.max_q = batch->max_q;
  a.sched.group = n_q_heads / cache->n_kv_heads;
  a.sched.n_kv = cache->n_kv_heads;
  a.sched.rows = p.rows;
  a.sched.pitch = p.pitch;
  a.sched.tile = p.tile;
  a.sched.extra = p.extra;
  a.sched.min_len = p.extra + 2;
  a.out.O = static_cast<__nv_bfloat16*>(O);
  a.out.ldo = ldo;
  a.out.lse = lse;
  a.out.n_q_heads = n_q_heads;
  a.parts = kv_parts(static_cast<uint8_t*>(ws) + kStatusBytes, p.workers, p.pitch);
  a.scale = scale;
  a.status = static_cast<int32_t*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool i8 = (cache->flags & MQ_KV_INT8) != 0;
  int e;
  if (p.chunk) e = launch_kv_chunk(a, cache->head_dim, i8, p.workers, st);
  else if (cache->head_dim == 128) e = i8 ? launch_decode<128, true>(a, p.workers, st) : launch_decode<128, false>(a, p.workers, st);
  else e = i8 ? launch_decode<64, true>(a, p.workers, st) : launch_decode<64, false>(a, p.workers, st);
  if (e != MQ_OK) return e;
  return launch_kv_combine(a.sched, a.parts, a.out, p.workers, cache->head_dim, st);
}
