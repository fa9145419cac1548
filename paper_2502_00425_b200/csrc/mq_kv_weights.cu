// The softmax weight every cached key receives from a chunk's rows, accumulated:
//   W_out[b, g, j] = W_in[b, g, j] + sum over rows i and heads h that see j of exp(scale * Q[i, h] . K[j, g] - lse[i, h])
// lse (the log of every row's softmax denominator) comes from the attention call, so one pass over K suffices.
//
// This is the kernel for few query rows (decode steps), bound by reading K; chunks take mq_kv_weights_chunk.cu.  Like the
// decode attention it lets every warp stream 16 keys at a time into a ring of its own and multiply them as the rows of
// the instruction's tile: a key's sum is over the columns, registers of four neighbouring lanes, and is written once.
// The work line is the sequences' key tiles, cut into equal ranges; nothing has to be joined.  No atomics, one order of
// summation.  One token of 32 sequences of 256 to 4096 keys, 4 heads of 128: 14.7 us for 48 MB of keys (3.3 TB/s; the
// pass is too short for more: launch, work line and the first loads are 5 us of it).  More than 8 kN rows (only where a group does not fit the chunk kernel) are walked in blocks per key tile.
#include "mq_kv_warp.cuh"
#include "mq_kv_weights.cuh"

namespace mq {
namespace {

constexpr int kWarps = kStreamWarps, kThreads = kStreamThreads, kTile = kStreamTile;
// Query rows per key/value head (tokens x heads of the group) up to which a call comes here.  This kernel / the chunk kernel
// in us, 4 heads of 128 in bf16: 14 rows over 1 x 2000 keys 6.2 / 7.5, over 16 x 8000 36 / 80; 28 rows 11.0 / 7.5 and
// 86 / 80; 56 rows 16 / 7.6 and 150 / 80.
constexpr int kFewRows = 16;
constexpr int kExtra = 2;      // what a unit costs besides its tiles (its queries), in tiles

template <int kD, bool kI8, int kN>
struct Cfg {
  static constexpr int kStage = KeyTile<kD, kI8>::kBytes;
  static constexpr int kStages = kStage == 4096 ? 3 : 4;
  static constexpr int kCtas = 4;
  static constexpr int kRing = kStage * kStages;
  static constexpr int kSmem = 1024 + kWarps * kRing;
};

template <int kD, bool kI8, int kN>
__global__ void __launch_bounds__(kThreads, (Cfg<kD, kI8, kN>::kCtas))
kv_weights_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ WeightParams p) {
  using C = Cfg<kD, kI8, kN>;
  using T = KeyTile<kD, kI8>;
  constexpr int kRows = 8 * kN;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[kWarps][C::kStages];
  __shared__ int64_t red[kWarps];
  __shared__ int abort_flag;
  __shared__ int32_t status[2];
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + kWarps * C::kRing);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2, t4 = lane & 3;
  if (tid == 0) {
    abort_flag = 0;
    status[0] = status[1] = MQ_OK;
    for (int i = 0; i < kWarps * C::kStages; ++i) mbar_init(&full[0][0] + i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_launch_dependents();
  pdl_wait();

  // length of a head's stretch of the line (all of a sequence's heads are alike), summed over the sequences before each one
  auto stretch = [&](const KvSeq& s) -> int { return s.n_all > 0 ? (s.n_all + kTile - 1) / kTile + kExtra : 0; };
  const int n = p.b.n_seq;
  {
    const int per = (n + kThreads - 1) / kThreads;
    int64_t sum = 0;
    for (int k = 0; k < per; ++k) {
      const int b = tid * per + k;
      if (b >= n) break;
      sum += (int64_t)stretch(kv_seq(p.b, p.c.page_shift, p.max_q, b)) * p.c.n_kv_heads;
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
  const int64_t total = prefix[n];
  const int64_t share = total >> 31 ? (total + gridDim.x - 1) / gridDim.x : (int64_t)(((uint32_t)total + gridDim.x - 1u) / gridDim.x);
  int64_t at = min(total, (int64_t)blockIdx.x * share);
  const int64_t stop = min(total, at + share);
  const uint32_t ring = kv_smem_u32(smem) + (uint32_t)(warp * C::kRing);
  uint32_t asked = 0, taken = 0;
  bool ok = true;
  while (ok && at < stop) {
    int b = 0, hi = n;   // prefix[b] <= at < prefix[hi]
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (prefix[mid] <= at) b = mid;
      else hi = mid;
    }
    const KvSeq s = kv_seq(p.b, p.c.page_shift, p.max_q, b);
    const int per_head = stretch(s);
    const int64_t x = at - prefix[b];
    const int g = (int)(x >> 31 ? x / per_head : (int64_t)((uint32_t)x / (uint32_t)per_head)), skip = (int)(x - (int64_t)g * per_head);
    const int len = (int)min((int64_t)(per_head - skip), stop - at);
    at += len;
    const int t0 = max(0, skip - kExtra), t1 = max(0, skip + len - kExtra);
    if (t0 == t1) continue;
    const int ctx = s.n_all - s.n_new;
    const int32_t *table = p.b.page_table + (int64_t)b * p.b.max_pages, *perm = p.b.perm ? p.b.perm + s.begin : nullptr;
    const int first_key = (t0 * kWarps + warp) * 16;
    const int n_my = min(t1 - t0, s.n_all > first_key ? (s.n_all - first_key + kTile - 1) / kTile : 0);
    PageWindow pages(table, first_key, p.c.page_shift, n_my, lane);
    auto ask = [&](int i) {
      if (i >= n_my) return;
      int page = pages.page(i, lane);
      if (lane == 0) {
        if ((unsigned)page >= (unsigned)p.c.n_pages) {
          page = max(p.c.n_pages, 1);   // a page number the map does not have: zeros
          if (p.status) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
        }
        const int st = (int)(asked % C::kStages), slot = (first_key + i * kTile) & ((1 << p.c.page_shift) - 1);
        mbar_arrive_expect_tx(&full[warp][st], C::kStage);
        T::load(ring + (uint32_t)(st * C::kStage), &tmap_k, slot, g, page, &full[warp][st]);
      }
      ++asked;
    };

    // ---- a block of query rows: operands, what turns scores into log2 units, log-sum-exps (log2 units), and sight
    const int n_rows = s.n_new * p.group.d, blocks = (n_rows + kRows - 1) / kRows;
    const float base_fac = p.scale * 1.4426950408889634f * (kI8 ? p.c.k_scale[g] : 1.0f);
    uint32_t qf[kN][kD / 16][2];
    float fac[kN][2], nl[kN][2];
    int lim[kN][2], all_see = INT_MAX;   // every row of the block sees the keys below all_see
    auto fetch_rows = [&](int row0) {
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        const int r = row0 + 8 * nt + quad, tok = r / p.group;
        fetch_query<kD, kI8>(p.Q + (int64_t)(s.begin + tok) * p.ldq + (int64_t)(g * p.group.d + r - tok * p.group.d) * (kD * 2), r < n_rows, t4, qf[nt]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int rr = row0 + 8 * nt + 2 * t4 + e, tk = rr / p.group;
          const bool live = rr < n_rows;
          const float l = live ? p.lse[(int64_t)(s.begin + tk) * p.n_q_heads + g * p.group.d + rr - tk * p.group.d] : INFINITY;
          nl[nt][e] = l;
          lim[nt][e] = !live ? INT_MIN : perm ? perm[tk] : ctx + tk + 1;
        }
      }
      all_see = row0 + kRows > n_rows ? INT_MIN : perm ? ctx : ctx + row0 / p.group + 1;
    };
    auto finish_rows = [&]() {
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        finish_query<kD, kI8>(t4, base_fac, qf[nt], fac[nt]);
#pragma unroll
        for (int e = 0; e < 2; ++e)   // (a row that sees nothing has -inf and adds nothing)
          nl[nt][e] = fabsf(nl[nt][e]) == INFINITY ? -INFINITY : nl[nt][e] * -1.4426950408889634f;
      }
    };
    if (blocks > 0) fetch_rows(0);
#pragma unroll
    for (int i = 0; i < C::kStages - 1; ++i) ask(i);
    if (blocks > 0) finish_rows();

    for (int i = 0; i < n_my; ++i) {
      ask(i + C::kStages - 1);
      const int st = (int)(taken % C::kStages), key0 = first_key + i * kTile;
      // what the two keys of this lane had (asked for before the wait)
      const int ka = key0 + quad, kb = ka + 8;
      const int64_t out = (int64_t)b * p.seq_stride + (int64_t)g * p.head_stride;
      float old_a = 0.0f, old_b = 0.0f;
      if (t4 == 0 && p.W_in) {
        if (ka < min(ctx, p.w_keys)) old_a = p.W_in[out + ka];
        if (kb < min(ctx, p.w_keys)) old_b = p.W_in[out + kb];
      }
      if (!(ok = warp_all(mbar_wait(&full[warp][st], (taken / C::kStages) & 1u, &abort_flag, status, 91)))) break;
      ++taken;
      float sum_a = 0.0f, sum_b = 0.0f;
      for (int blk = 0; blk < blocks; ++blk) {
        if (blocks > 1) {
          fetch_rows(blk * kRows);
          finish_rows();
        }
        float sc[kN][4];
        key_scores<kD, kI8, kN>(ring + (uint32_t)(st * C::kStage), lane, qf, sc);
        const bool masked = key0 + 16 > all_see;
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = kv_exp2(fmaf(sc[nt][e], fac[nt][e & 1], nl[nt][e & 1]));
            if (masked) {
              const int key = e < 2 ? ka : kb, lm = lim[nt][e & 1];
              const bool sees = lm != INT_MIN && key < s.n_all && (perm ? key < ctx || perm[key - ctx] <= lm : key < lm);
              if (!sees) v = 0.0f;
            }
            if (e < 2) sum_a += v;
            else sum_b += v;
          }
      }
      sum_a += __shfl_xor_sync(0xffffffffu, sum_a, 1); sum_a += __shfl_xor_sync(0xffffffffu, sum_a, 2);
      sum_b += __shfl_xor_sync(0xffffffffu, sum_b, 1); sum_b += __shfl_xor_sync(0xffffffffu, sum_b, 2);
      if (t4 == 0) {
        if (ka < min(s.n_all, p.w_keys)) p.W_out[out + ka] = old_a + sum_a;
        if (kb < min(s.n_all, p.w_keys)) p.W_out[out + kb] = old_b + sum_b;
        if (max(ka, kb) >= p.w_keys && min(ka, kb) < s.n_all && s.n_all > p.w_keys && p.status) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
      }
      __syncwarp();   // every lane has read the tile before its slot is asked to be filled again
    }
  }
  if (!ok) {
    for (; taken < asked; ++taken) mbar_wait_drain(&full[warp][taken % C::kStages], (taken / C::kStages) & 1u, 20000ull);
    if (lane == 0 && p.status && atomicCAS(p.status, MQ_OK, MQ_ERR_TIMEOUT) == MQ_OK) p.status[1] = 91;
  }
}

template <int kD, bool kI8, int kN>
int launch(const WeightParams& p, int64_t most, cudaStream_t st) {
  using C = Cfg<kD, kI8, kN>;
  const size_t smem = C::kSmem + ((size_t)p.b.n_seq + 1) * sizeof(int64_t);
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_weights_kernel<kD, kI8, kN>, C::kSmem + (kMaxKvSeqs + 1) * (int)sizeof(int64_t))) return MQ_ERR_CUDA;
  CUtensorMap mk;
  // (a cache without pages: any address will do, nothing is read)
  if (!encode_key_tiles(&mk, p.c.K, reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(p.W_out) & ~uintptr_t(15)), p.c, kD, kI8)) return MQ_ERR_CUDA;
  const int64_t cap = (int64_t)sm_count() * C::kCtas;
  const cudaError_t e = launch_pdl(kv_weights_kernel<kD, kI8, kN>, dim3((unsigned)(most < cap ? most : cap)), dim3(kThreads), smem, st, mk, p);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" int mq_kv_weights(const void* Q, int64_t ldq, const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads,
                             float scale, const float* lse, const float* W_in, float* W_out, int64_t w_seq_stride,
                             int64_t w_head_stride, int32_t w_keys, int32_t* status, void* stream) {
  WeightParams p{};
  int rc = check_kv_cache(cache, &p.c);
  if (rc != MQ_OK) return rc;
  if ((rc = check_kv_batch(batch, &p.b)) != MQ_OK) return rc;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads) return MQ_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || !std::isfinite(scale)) return MQ_ERR_INVALID_ARG;
  const int64_t reach = (int64_t)batch->max_pages * cache->page_size;
  const int group = n_q_heads / cache->n_kv_heads;
  if (ldq < (int64_t)n_q_heads * cache->head_dim || w_head_stride < 0 || w_seq_stride < 0 || w_keys < 0) return MQ_ERR_INVALID_ARG;
  if ((int64_t)batch->max_q * group > (1 << 30)) return MQ_ERR_UNSUPPORTED;
  if (batch->n_seq == 0 || reach == 0 || w_keys == 0) return MQ_OK;
  if (!W_out || (batch->total_q > 0 && (!Q || !lse))) return MQ_ERR_INVALID_ARG;
  // heads or sequences that share entries of W_out would write them at the same time
  const int64_t stride[2] = {w_head_stride, w_seq_stride}, count[2] = {cache->n_kv_heads, batch->n_seq};
  if (!kv_apart(w_keys < reach ? w_keys : reach, 2, stride, count)) return MQ_ERR_INVALID_ARG;
  if (!kv_aligned16(Q) || ldq % 8) return MQ_ERR_ALIGNMENT;
  p.Q = static_cast<const uint8_t*>(Q);
  p.ldq = ldq * 2;
  p.max_q = batch->max_q;
  p.group = fast_div(group);
  p.n_q_heads = n_q_heads;
  p.scale = scale;
  p.lse = lse;
  p.W_in = W_in;
  p.W_out = W_out;
  p.seq_stride = w_seq_stride;
  p.head_stride = w_head_stride;
  p.w_keys = w_keys;
  p.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool i8 = (cache->flags & MQ_KV_INT8) != 0;
  const int64_t rows = (int64_t)batch->max_q * group, units = (int64_t)batch->n_seq * cache->n_kv_heads;
  // (a token's heads have to fit into a row tile of the chunk kernel)
  if (rows > kFewRows && group <= 128) return launch_kv_weights_chunk(p, cache->head_dim, i8, units * ((reach + 127) / 128), st);
  const int64_t most = units * ((reach + kTile - 1) / kTile);
  if (rows <= 8) {
    if (cache->head_dim == 128) return i8 ? launch<128, true, 1>(p, most, st) : launch<128, false, 1>(p, most, st);
    return i8 ? launch<64, true, 1>(p, most, st) : launch<64, false, 1>(p, most, st);
  }
  if (cache->head_dim == 128) return i8 ? launch<128, true, 2>(p, most, st) : launch<128, false, 2>(p, most, st);
  return i8 ? launch<64, true, 2>(p, most, st) : launch<64, false, 2>(p, most, st);
}
