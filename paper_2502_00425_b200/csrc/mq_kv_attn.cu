// Attention of the new tokens of a ragged batch over a paged key/value cache.
//
//   O[i, h] = sum_j P[i, j] V[j, g],  P = softmax_j(scale * Q[i, h] . K[j, g]),  lse = log of the denominator
//
// The kernel of this file is the one for few query rows (decode steps): it is bound by reading K and V once.  A unit is 8
// or 16 query rows (tokens x the query heads of one key/value head), so a key is read once for the whole group.
//   * A warp is on its own: it streams 16 keys at a time (K and V rows by TMA straight from the pages, one lane asking, two or
//     more tiles in flight) into its own ring in shared memory and runs a complete online softmax over them on
//     mma.sync; there is no block-wide barrier until the four warps' results are joined at the end of a range.
//     Tensor-core throughput is no concern here: at the cache's rate an SM sees 16 keys in about 190 cycles.
//   * Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T: the 16 keys, and 16 channels, are the rows of the
//     instruction's tile and the query rows its 8 columns, so a group of up to 8 heads wastes nothing.  P^T changes from
//     the layout of a result to that of an operand by an 8 x 8 transpose in registers.
//   * The exponents are taken relative to the running maximum, the accumulator is rescaled only when a row's maximum moved.  The
//     probabilities are rounded once, to the values' type, as operands of mma.sync have to be; the sums take them unrounded.
//   * An int8 cache is read as codes and widened in registers to fp16 exactly (the products' sums do not care in which
//     order the channels come, so a thread takes contiguous codes); the scales multiply the scores and the result.
//     Queries are scaled by a power of two per row: fp16 then holds all bits of channels down to 2^-31 of the row's largest.
// 64 sequences of 64 to 8192 keys, 8 key/value heads of 128, groups of 4: 78 us in bf16 (449 MB, 5.8 TB/s, 88 % of a plain
// copy) and 50 us in int8 (225 MB, 4.5 TB/s).  There 446 warp instructions go with 16 keys, all counted; issue is busy for 54 %
// of the cycles in which an SM has work (integer pipe 47 %), three warps to a scheduler wait most for the fixed latencies
// of their own chains, and 13 % of the time an SM has no work (start, and ranges that end early).  Two blocks of 8 rows
// spill 132 bytes in int8.  One sequence of 3361 keys: 9 us, of which the two launches are half.
#include "mq_kv_warp.cuh"

namespace mq {
namespace {

constexpr int kWarps = kStreamWarps, kThreads = kStreamThreads, kTile = kStreamTile;
constexpr int kExtra = 4;         // what a unit costs besides its tiles, in tiles (64 ragged int8 sequences: 59 us with 2, 50 with 4, 54 with 8)
constexpr int kMinLen = 2;        // a worker's least share of the line (one sequence of 3361 keys: 9.0 us with 2, 11.7 with 6)
// fp16 probabilities reach down to 2^-24 only: with the reference 14 below the maximum they run up to 2^14 instead of 1, and
// what is lost below is 2^-39 of the largest one (a sum over them stays in float32 either way).
constexpr float kLiftF16 = 14.0f;

// kN: query rows of a unit, in eights
template <int kD, bool kI8, int kN>
struct Cfg {
  static constexpr int kRows = 8 * kN;
  static constexpr int kStage = 2 * KeyTile<kD, kI8>::kBytes;   // K and V of 16 keys
  // three CTAs with two stages of 8 KB (78.4 us in the case above) rather than two with three (79.6 us); 4 KB stages have
  // room for four
  static constexpr int kCtas = kStage == 8192 && kN == 2 ? 2 : 3;   // per SM
  static constexpr int kStages = kStage == 8192 && kN == 1 ? 2 : kStage == 8192 ? 3 : 4;
  static constexpr int kRing = kStage * kStages;
  static constexpr int kPitch = kD + 4;                  // floats between rows of the warps' results
  static constexpr int kSmem = 1024 + kWarps * kRing;    // (swizzled tiles stand on 1024-byte boundaries)
  static_assert(kWarps * kRing >= kWarps * kRows * kPitch * 4, "the join of the warps reuses the rings");
};
constexpr int decode_ctas(int dim, bool i8, int n) {
  return dim == 128 ? (i8 ? (n == 1 ? Cfg<128, true, 1>::kCtas : Cfg<128, true, 2>::kCtas) : (n == 1 ? Cfg<128, false, 1>::kCtas : Cfg<128, false, 2>::kCtas))
                    : (i8 ? (n == 1 ? Cfg<64, true, 1>::kCtas : Cfg<64, true, 2>::kCtas) : (n == 1 ? Cfg<64, false, 1>::kCtas : Cfg<64, false, 2>::kCtas));
}

template <int kD, bool kI8, int kN>
__global__ void __launch_bounds__(kThreads, (Cfg<kD, kI8, kN>::kCtas))
kv_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ KvAttnArgs p) {
  using C = Cfg<kD, kI8, kN>;
  using T = KeyTile<kD, kI8>;
  constexpr int kSteps = kD / 16, kRows = C::kRows;
  constexpr float kLift = kI8 ? kLiftF16 : 0.0f;   // m: the exponents' reference, the running maximum less this
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[kWarps][C::kStages];   // a tile has landed
  __shared__ int abort_flag;
  __shared__ float ml_s[kWarps][kRows][2];
  __shared__ int64_t red[kWarps];
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + kWarps * C::kRing);
  KvSeq* seqs = reinterpret_cast<KvSeq*>(prefix + p.sched.b.n_seq + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, t4 = lane & 3;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < kWarps * C::kStages; ++i) mbar_init(&full[0][0] + i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_launch_dependents();
  pdl_wait();
  const KvSchedArgs& sc = p.sched;
  sched_prefix<kThreads>(sc, prefix, red, seqs);
  const int64_t total = prefix[sc.b.n_seq];
  const int64_t share = sched_share(sc, total, gridDim.x);
  KvRecord rec{};
  int64_t at = min(total, (int64_t)blockIdx.x * share);
  const int64_t stop = min(total, at + share);
  const uint32_t ring = kv_smem_u32(smem) + (uint32_t)(warp * C::kRing);
  uint32_t asked = 0, taken = 0;   // tiles of this warp so far (ring positions and phases run on over units)
  bool ok = true;
  while (at < stop) {
    const KvUnit u = sched_unit(sc, prefix, at, seqs);
    const int len = (int)min((int64_t)(u.tiles + sc.extra - u.skip), stop - at);   // of this range on the line
    const int t0 = max(0, u.skip - sc.extra), t1 = max(0, u.skip + len - sc.extra);
    const int64_t unit_at = at - u.skip;
    at += len;
    if (t0 == t1) continue;   // the range ends before the unit's first tile
    const int end = sched_end(sc, u.s, u.rb), ctx = u.s.n_all - u.s.n_new;
    const int row0 = u.rb * kRows, n_rows = min(kRows, u.s.n_new * sc.group.d - row0);
    const int32_t* table = sc.b.page_table + (int64_t)u.b * sc.b.max_pages;

    // ---- the warp's stream of tiles: tile t holds keys (t * kWarps + warp) * 16 ..; tiles behind the last key are not asked for
    const int first_key = (t0 * kWarps + warp) * 16;
    const int n_my = min(t1 - t0, end > first_key ? (end - first_key + kTile - 1) / kTile : 0);
    PageWindow pages(table, first_key, p.cache.page_shift, n_my, lane);
    // query operands (column quad of block nt is row 8 nt + quad of the unit) and scales: asked for here, used below
    uint32_t qf[kN][kSteps][2];
#pragma unroll
    for (int nt = 0; nt < kN; ++nt) {
      const int r = row0 + 8 * nt + quad, tok = r / sc.group;
      fetch_query<kD, kI8>(p.Q + (int64_t)(u.s.begin + tok) * p.ldq + (int64_t)(u.g * sc.group.d + r - tok * sc.group.d) * (kD * 2), 8 * nt + quad < n_rows, t4, qf[nt]);
    }
    const float k_scale = kI8 ? p.cache.k_scale[u.g] : 1.0f, v_scale = kI8 ? p.cache.v_scale[u.g] : 1.0f;
    auto ask = [&](int i) {
      if (i >= n_my) return;
      int page = pages.page(i, lane);
      if (lane == 0) {
        if ((unsigned)page >= (unsigned)p.cache.n_pages) {
          page = max(p.cache.n_pages, 1);   // a page number the maps do not have: zeros
          atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
        }
        const int s = (int)(asked % C::kStages), slot = (first_key + i * kTile) & ((1 << p.cache.page_shift) - 1);
        const uint32_t dst = ring + (uint32_t)(s * C::kStage);
        mbar_arrive_expect_tx(&full[warp][s], C::kStage);
        T::load(dst, &tmap_k, slot, u.g, page, &full[warp][s]);
        T::load(dst + T::kBytes, &tmap_v, slot, u.g, page, &full[warp][s]);
      }
      ++asked;
    };
#pragma unroll
    for (int i = 0; i < C::kStages - 1; ++i) ask(i);

    float fac[kN][2];               // scores -> log2 units, rows 2 t4 and 2 t4 + 1 of block nt
    int lim[kN][2];                 // how far these rows see: without perm, keys below lim; with it, the context and the chunk's
                                    // rows whose index is at most lim
    const int32_t* perm = sc.b.perm ? sc.b.perm + u.s.begin : nullptr;
#pragma unroll
    for (int nt = 0; nt < kN; ++nt) {
      finish_query<kD, kI8>(t4, p.scale * 1.4426950408889634f * k_scale, qf[nt], fac[nt]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * nt + 2 * t4 + e, tk = (row0 + rr) / sc.group;
        lim[nt][e] = rr >= n_rows ? INT_MIN : perm ? perm[tk] : ctx + tk + 1;
      }
    }
    const int all_see = perm ? ctx : min(end, ctx + row0 / sc.group + 1);   // every row of the unit sees the keys below
    auto sees = [&](int key, int lm) -> bool {
      if (key >= end || lm == INT_MIN) return false;
      if (!perm) return key < lm;
      return key < ctx || perm[key - ctx] <= lm;
    };

    float o[kSteps][kN][4];    // O^T: channels 16 mt + quad (+ 8) x rows 2 t4, 2 t4 + 1 of block nt
    float m[kN][2], l[kN][2];
#pragma unroll
    for (int nt = 0; nt < kN; ++nt) {
#pragma unroll
      for (int mt = 0; mt < kSteps; ++mt) o[mt][nt][0] = o[mt][nt][1] = o[mt][nt][2] = o[mt][nt][3] = 0.0f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.0f;
    }

    for (int i = 0; i < n_my; ++i) {
      ask(i + C::kStages - 1);
      const int stage = (int)(taken % C::kStages);
      if (!(ok = warp_all(mbar_wait(&full[warp][stage], (taken / C::kStages) & 1u, &abort_flag, p.status, 90)))) break;
      ++taken;
      const uint32_t kt = ring + (uint32_t)(stage * C::kStage), vt = kt + T::kBytes;
      const int key0 = first_key + i * kTile;
      {
        float s[kN][4];
        key_scores<kD, kI8, kN>(kt, lane, qf, s);
        if (!kI8 && key0 + 16 > end) {
          // slots behind the last key hold anything: their values must not meet the zeros of P as infinities
#pragma unroll
          for (int c = 0; c < 16 * kD / 8 / 32; ++c) {
            const int idx = c * 32 + lane, r = idx / (kD / 8), pc = idx % (kD / 8);
            if (key0 + r >= end) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vt + T::piece(r, pc)), "r"(0) : "memory");
          }
          fence_proxy_async_smem();   // (the slot's next tile is written by TMA)
          __syncwarp();
        }
        const bool masked = key0 + 16 > all_see;
        unsigned seen = ~0u;   // bit 4 nt + e: score s[nt][e] counts
        if (masked) {
          seen = 0u;
#pragma unroll
          for (int nt = 0; nt < kN; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (sees(key0 + quad + 8 * (e >> 1), lim[nt][e & 1])) seen |= 1u << (4 * nt + e);
        }
        bool grown = false;
        float top[kN][2];
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[nt][e] *= fac[nt][e & 1];
            if (masked && !((seen >> (4 * nt + e)) & 1u)) s[nt][e] = -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = fmaxf(s[nt][e], s[nt][e + 2]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            top[nt][e] = x - kLift;
            grown |= top[nt][e] > m[nt][e];
          }
        }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
          for (int nt = 0; nt < kN; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float n = fmaxf(m[nt][e], top[nt][e]);
              const float f = m[nt][e] == -INFINITY ? 0.0f : kv_exp2(m[nt][e] - n);
              m[nt][e] = n;
              l[nt][e] *= f;
#pragma unroll
              for (int mt = 0; mt < kSteps; ++mt) { o[mt][nt][e] *= f; o[mt][nt][e + 2] *= f; }
            }
        }
        uint32_t pf[kN][2];
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
          // (a row without keys yet: exp2(-inf) = 0)
          const float u0 = m[nt][0] == -INFINITY ? 0.0f : m[nt][0], u1 = m[nt][1] == -INFINITY ? 0.0f : m[nt][1];
          s[nt][0] = kv_exp2(s[nt][0] - u0); s[nt][1] = kv_exp2(s[nt][1] - u1);
          s[nt][2] = kv_exp2(s[nt][2] - u0); s[nt][3] = kv_exp2(s[nt][3] - u1);
          l[nt][0] += s[nt][0] + s[nt][2];
          l[nt][1] += s[nt][1] + s[nt][3];
          pf[nt][0] = mat_transpose(kI8 ? kv_pack_f16(s[nt][0], s[nt][1]) : kv_pack_bf16(s[nt][0], s[nt][1]));
          pf[nt][1] = mat_transpose(kI8 ? kv_pack_f16(s[nt][2], s[nt][3]) : kv_pack_bf16(s[nt][2], s[nt][3]));
        }
        // A value that some rows may not see must not reach them even if it is infinite or NaN (0 * inf): such a tile
        // is multiplied key by key.  Only tiles with rows of different sight can hold one.
        bool odd = false;
        if (!kI8 && masked && all_see < end) {
          uint32_t big = 0u;
#pragma unroll
          for (int c = 0; c < T::kBytes / 512; ++c) {
            uint32_t x[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(vt + (uint32_t)(c * 32 + lane) * 16u));
#pragma unroll
            for (int w = 0; w < 4; ++w) big = __vmaxu2(big, x[w] & 0x7fff7fffu);
          }
          odd = __any_sync(0xffffffffu, (big & 0xffffu) >= 0x7f80u || (big >> 16) >= 0x7f80u);
        }
        if (!kI8 && odd) {
#pragma unroll 1
          for (int key = 0; key < 16; ++key) {
            const int from = ((key & 7) << 2) | t4;
#pragma unroll
            for (int nt = 0; nt < kN; ++nt) {
              const float a0 = __shfl_sync(0xffffffffu, s[nt][0], from), a1 = __shfl_sync(0xffffffffu, s[nt][1], from);
              const float b0 = __shfl_sync(0xffffffffu, s[nt][2], from), b1 = __shfl_sync(0xffffffffu, s[nt][3], from);
              const unsigned vis = __shfl_sync(0xffffffffu, seen, from) >> (4 * nt + (key < 8 ? 0 : 2));
              const float p0 = key < 8 ? a0 : b0, p1 = key < 8 ? a1 : b1;
#pragma unroll
              for (int mt = 0; mt < kSteps; ++mt)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                  unsigned short x;
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(vt + T::piece(key, 2 * mt + hh) + (uint32_t)quad * 2u));
                  const float v = __uint_as_float((uint32_t)x << 16);
                  if (vis & 1u) o[mt][nt][2 * hh] = fmaf(p0, v, o[mt][nt][2 * hh]);
                  if (vis & 2u) o[mt][nt][2 * hh + 1] = fmaf(p1, v, o[mt][nt][2 * hh + 1]);
                }
            }
          }
        } else if (!kI8) {
#pragma unroll
          for (int mt = 0; mt < kSteps; ++mt) {
            uint32_t a[4];
            ldsm_x4_trans(vt + T::piece((lane & 7) + ((lane >> 4) << 3), 2 * mt + ((lane >> 3) & 1)), a);
#pragma unroll
            for (int nt = 0; nt < kN; ++nt) mma_16816<false>(o[mt][nt], a, pf[nt][0], pf[nt][1]);
          }
        } else {
          // result row quad (+ 8) of product mt is channel quad * D/8 + 2 mt (+ 1): a thread reads D/8 contiguous codes of each of its
          // four keys
          constexpr int kWords = kD / 32;
          uint32_t x[4][kWords];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = 2 * t4 + (r & 1) + 8 * (r >> 1);
            if (kD == 128)
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(x[r][0]), "=r"(x[r][1]), "=r"(x[r][2 % kWords]), "=r"(x[r][3 % kWords]) : "r"(vt + T::piece(key, quad)));
            else
              asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];"
                           : "=r"(x[r][0]), "=r"(x[r][1]) : "r"(vt + T::piece(key, quad >> 1) + (uint32_t)(quad & 1) * 8u));
          }
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            uint32_t a[2][4];   // two products: channels 4 w, 4 w + 1 and 4 w + 2, 4 w + 3 of this thread's run
            i8x4_to_f16(__byte_perm(x[0][w], x[1][w], 0x5140), a[0][0], a[0][1]);
            i8x4_to_f16(__byte_perm(x[2][w], x[3][w], 0x5140), a[0][2], a[0][3]);
            i8x4_to_f16(__byte_perm(x[0][w], x[1][w], 0x7362), a[1][0], a[1][1]);
            i8x4_to_f16(__byte_perm(x[2][w], x[3][w], 0x7362), a[1][2], a[1][3]);
#pragma unroll
            for (int nt = 0; nt < kN; ++nt) {
              mma_16816<true>(o[2 * w][nt], a[0], pf[nt][0], pf[nt][1]);
              mma_16816<true>(o[2 * w + 1][nt], a[1], pf[nt][0], pf[nt][1]);
            }
          }
        }
      }
      __syncwarp();   // every lane has read the tile before its slot is asked to be filled again
    }
#pragma unroll
    for (int nt = 0; nt < kN; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 4);
        l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 8);
        l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 16);
      }

    // ---- join the warps: each ran a softmax over its own keys
    if (__syncthreads_or(!ok)) {   // (the rings are free)
      ok = false;
      break;
    }
    float* join = reinterpret_cast<float*>(smem) + warp * (kRows * C::kPitch);
#pragma unroll
    for (int nt = 0; nt < kN; ++nt) {
      const int r = 8 * nt + 2 * t4;
      if (quad == 0) {
        ml_s[warp][r][0] = m[nt][0]; ml_s[warp][r][1] = l[nt][0];
        ml_s[warp][r + 1][0] = m[nt][1]; ml_s[warp][r + 1][1] = l[nt][1];
      }
#pragma unroll
      for (int mt = 0; mt < kSteps; ++mt) {
        const int d0 = kI8 ? quad * (kD / 8) + 2 * mt : 16 * mt + quad, d1 = kI8 ? d0 + 1 : d0 + 8;
        join[r * C::kPitch + d0] = o[mt][nt][0];
        join[(r + 1) * C::kPitch + d0] = o[mt][nt][1];
        join[r * C::kPitch + d1] = o[mt][nt][2];
        join[(r + 1) * C::kPitch + d1] = o[mt][nt][3];
      }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == u.tiles;
    const int slot = 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0);
    constexpr int kColThreads = kD / 2;                 // two channels per thread
    const int col = ((int)threadIdx.x % kColThreads) * 2;
    for (int r = (int)threadIdx.x / kColThreads; r < n_rows; r += kThreads / kColThreads) {
      float mm = ml_s[0][r][0];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, ml_s[w][r][0]);
      float ll = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float mw = ml_s[w][r][0];
        const float f = mw == -INFINITY ? 0.0f : kv_exp2(mw - mm);
        ll = fmaf(f, ml_s[w][r][1], ll);
        const float2 v = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(smem) + (w * kRows + r) * C::kPitch + col);
        if (f != 0.0f) { x = fmaf(f, v.x, x); y = fmaf(f, v.y, y); }
      }
      if (whole) {
        const int tk = (row0 + r) / sc.group, tok = u.s.begin + tk, head = u.g * sc.group.d + (row0 + r) - tk * sc.group.d;
        const float inv = ll == 0.0f ? 0.0f : v_scale / ll;
        *reinterpret_cast<__nv_bfloat162*>(p.out.O + (int64_t)tok * p.out.ldo + (int64_t)head * kD + col) =
            __floats2bfloat162_rn(x * inv, y * inv);
        if (col == 0 && p.out.lse)
          p.out.lse[(int64_t)tok * p.out.n_q_heads + head] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * 0.6931471805599453f;
      } else {
        if (col == 0) p.parts.ml[(int64_t)slot * kRows + r] = make_float2(mm, ll);
        *reinterpret_cast<float2*>(p.parts.o + ((int64_t)slot * kRows + r) * kD + col) = make_float2(x * v_scale, y * v_scale);
      }
    }
    if (t0 == 0 && !whole) {
      // the pieces end with the worker whose range holds the unit's last tile
      const int64_t last = unit_at + sc.extra + u.tiles - 1;
      rec.n_parts = (last >> 31 ? (int)(last / share) : (int)((uint32_t)last / (uint32_t)share)) - (int)blockIdx.x + 1;
      rec.begin = u.s.begin; rec.row0 = row0; rec.n_rows = n_rows; rec.g = u.g;
    }
    fence_proxy_async_smem();   // (the rings are next written by TMA)
    __syncthreads();   // the join has been read before the next range fills the rings
  }
  if (!ok) {   // copies still landing in this CTA's shared memory get time to finish before it exits
    for (; taken < asked; ++taken) mbar_wait_drain(&full[warp][taken % C::kStages], (taken / C::kStages) & 1u, 20000ull);
    rec = KvRecord{};
  }
  if (threadIdx.x == 0) p.parts.rec[blockIdx.x] = rec;
}

// Joins the pieces of the units that are split.  kWarps warps share a row and take every kWarps-th piece: four where
// a unit has few rows and may have tens of pieces (a decode step of one sequence is as long as this chain of loads),
// one where it has 128 rows and mostly two pieces.  The record holds all that is needed: one dependent load before
// the pieces.
// Blocks of 512 threads where a row has one warp: most blocks find nothing to join, and starting them is what they cost (144
// whole units of 5 tiles: 25.2 us with 256 threads, 22.9 with 512, 24.0 with 1024).  Four warps to a row: 256 (one sequence of 3361 keys 9.3 us, 9.5 with 512).
template <int kWarpsPerRow>
constexpr int kJoinThreads = kWarpsPerRow > 1 ? 256 : 512;
template <int kD, int kWarpsPerRow>
__global__ void __launch_bounds__(kJoinThreads<kWarpsPerRow>)
kv_combine_kernel(const int pitch, const FastDiv group, const KvParts parts, const KvOutArgs out) {
  constexpr int kPer = kD / 32, kRows = kJoinThreads<kWarpsPerRow> / 32 / kWarpsPerRow;
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
      // (a reference of -inf: nothing but zeros, or scores that are all NaN, whose sum says so and is kept)
      const float back = m == -INFINITY ? 0.0f : kv_exp2(m - top);
      l *= back;
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] *= back;
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        const float f = ml[c].x == -INFINITY ? 0.0f : kv_exp2(ml[c].x - top);
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
      const float f = mk == -INFINITY ? 0.0f : kv_exp2(mk - m);
      l = fmaf(f, part[rr][k][kD + 1], l);
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] = fmaf(f, part[rr][k][lane * kPer + e], x[e]);
    }
  }
  if (!live) return;
  const int tk = (rec.row0 + r) / group, tok = rec.begin + tk, head = rec.g * group.d + (rec.row0 + r) - tk * group.d;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  __nv_bfloat16* dst = out.O + (int64_t)tok * out.ldo + (int64_t)head * kD + lane * kPer;
  if (kPer == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(kv_pack_bf16(x[0] * inv, x[1] * inv), kv_pack_bf16(x[2 % kPer] * inv, x[3 % kPer] * inv));
  else
    *reinterpret_cast<uint32_t*>(dst) = kv_pack_bf16(x[0] * inv, x[1] * inv);
  if (lane == 0 && out.lse)
    out.lse[(int64_t)tok * out.n_q_heads + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <int kD, bool kI8, int kN>
int launch_decode(const KvAttnArgs& a, int workers, cudaStream_t st) {
  using C = Cfg<kD, kI8, kN>;
  const size_t smem = C::kSmem + ((size_t)a.sched.b.n_seq + 1) * (sizeof(int64_t) + sizeof(KvSeq));
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_decode_kernel<kD, kI8, kN>, C::kSmem + (kMaxKvSeqs + 1) * (int)(sizeof(int64_t) + sizeof(KvSeq)))) return MQ_ERR_CUDA;
  CUtensorMap mk, mv;
  if (!encode_key_tiles(&mk, a.cache.K, a.Q, a.cache, kD, kI8) || !encode_key_tiles(&mv, a.cache.V, a.Q, a.cache, kD, kI8)) return MQ_ERR_CUDA;
  const cudaError_t e = launch_pdl(kv_decode_kernel<kD, kI8, kN>, dim3((unsigned)workers), dim3(kThreads), smem, st, mk, mv, a);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}
template <int kD, bool kI8>
int launch_decode(const KvAttnArgs& a, int workers, cudaStream_t st) {
  return a.sched.rows == 8 ? launch_decode<kD, kI8, 1>(a, workers, st) : launch_decode<kD, kI8, 2>(a, workers, st);
}

// Which kernel, and how many workers.  Up to kFewRows query rows per key/value head (tokens x heads of the group) take the
// kernel above in blocks of 8 or 16 rows, more take the 128-row tensor-memory kernel of mq_kv_chunk.cu.  Both in us, heads
// of 128, bf16, 4 key/value heads, this kernel / that one: 14 rows over 16 x 8000 keys 56 / 69, 28 rows over 1 x 2000
// 12 / 19, over 16 x 2000 30 / 31, over 16 x 8000 94 / 68; 56 rows 13 / 19, 47 / 31 and 164 / 68.  The lengths are not known
// on the host, so the rule is the rows at which the middle is a draw.
constexpr int kFewRows = 32;
struct Plan {
  bool chunk;
  int workers, rows, pitch, tile, extra;
};
Plan attn_plan(const mq_kv_batch* b, const mq_kv_cache* c, int group) {
  Plan p{};
  // (a token's heads have to fit into a block of that kernel)
  p.chunk = (int64_t)b->max_q * group > kFewRows && group <= 128;
  if (p.chunk) kv_chunk_shape(group, &p.rows, &p.pitch, &p.tile, &p.extra);
  else p.rows = p.pitch = (int64_t)b->max_q * group <= 8 ? 8 : 16, p.tile = kTile, p.extra = kExtra;
  const int64_t blocks = ((int64_t)b->max_q * group + p.rows - 1) / p.rows;
  const int64_t tiles = (((int64_t)b->max_pages * c->page_size) + p.tile - 1) / p.tile;
  const int64_t most = (int64_t)b->n_seq * c->n_kv_heads * blocks * (tiles > 0 ? tiles : 1);
  const int64_t cap = (int64_t)sm_count() * (p.chunk ? 1 : decode_ctas(c->head_dim, (c->flags & MQ_KV_INT8) != 0, p.rows / 8));
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
  // (a slot has as many rows as a sequence can have, at most)
  const int64_t rows = (int64_t)a.max_q * a.group.d < a.rows ? (int64_t)a.max_q * a.group.d : a.rows;
  constexpr int per = kJoinThreads<kW> / (kW * 32);
  return launch_pdl(kv_combine_kernel<kD, kW>, dim3((unsigned)workers, (unsigned)((rows + per - 1) / per)), dim3(kJoinThreads<kW>), 0, st,
                    a.pitch, a.group, parts, out);
}
}  // namespace

int launch_kv_combine(const KvSchedArgs& a, const KvParts& parts, const KvOutArgs& out, int workers, int dim, cudaStream_t st) {
  // Slots of few rows come in long chains (one sequence is spread over all workers): four warps share a row's chain.  With
  // one warp / four in us, the whole call: one token over 3361 keys 11.6 / 9.0, over 8 x 2000 13.2 / 13.7; a chunk of 40
  // tokens over 4000 keys (256-row slots) 24 / 39, of 2 x 1024 over 8000 256 / 308.
  const bool few = a.pitch <= 16;
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
  a.sched.group = fast_div(n_q_heads / cache->n_kv_heads);
  a.sched.by_rows = fast_div(p.rows);
  a.sched.n_kv = cache->n_kv_heads;
  a.sched.rows = p.rows;
  a.sched.pitch = p.pitch;
  a.sched.tile = p.tile;
  a.sched.tile_shift = 31 - __builtin_clz((unsigned)p.tile);
  a.sched.extra = p.extra;
  a.sched.min_len = p.chunk ? p.extra + 2 : kMinLen;
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
