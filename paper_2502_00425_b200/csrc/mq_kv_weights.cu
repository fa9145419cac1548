// The softmax weight every cached key receives from a chunk's rows, accumulated:
//   W_out[b, g, j] = W_in[b, g, j] + sum over rows i and heads h that see j of exp(scale * Q[i, h] . K[j, g] - lse[i, h])
// lse (the log of every row's softmax denominator) comes from the attention call, so one pass over K suffices.
//
// The product is taken with the KEYS as the rows of the tensor-core tile: a CTA owns 128 keys of one head (16 per
// warp), keeps them in registers as A fragments, and walks the query rows in blocks of 64; a key's sum is then over
// columns, i.e. over registers of four neighbouring lanes, and is written once.  No atomics, one order of summation.
// This is the kernel for few query rows, bound by reading K; chunks take mq_kv_weights_chunk.cu.
#include "mq_kv_weights.cuh"

namespace mq {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kKeys = kWarps * 16;   // keys of a CTA's tile
constexpr int kRowsQ = 64;           // query rows per step
constexpr int kFewRows = 64;         // up to here (tokens x heads of the group) this kernel, above the tensor-memory one

template <int kD>
struct Smem {
  static constexpr int kPitch = kD * 2 + 16;   // bytes between rows: neighbouring rows start in different banks
  static constexpr int kK = kKeys * kPitch;
  static constexpr int kQ = kRowsQ * kPitch;
  static constexpr int kBytes = kK + kQ + kRowsQ * 8;
};

template <int kD, bool kI8>
__global__ void __launch_bounds__(kThreads)
kv_weights_kernel(const __grid_constant__ WeightParams p) {
  using S = Smem<kD>;
  constexpr int kSteps = kD / 16, kPieces = kD / 8;   // 16-byte pieces of a bf16 row
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t red[kWarps];
  uint8_t* ks = smem;
  uint8_t* qs = smem + S::kK;
  float* row_lse = reinterpret_cast<float*>(qs + S::kQ);     // log2 units; +inf for a row that adds nothing
  int* row_lim = reinterpret_cast<int*>(row_lse + kRowsQ);
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + S::kBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2, t4 = lane & 3;
  pdl_launch_dependents();
  pdl_wait();

  // key tiles of the sequences before each one
  const int n = p.b.n_seq, per = (n + kThreads - 1) / kThreads;
  int64_t sum = 0;
  for (int k = 0; k < per; ++k) {
    const int b = tid * per + k;
    if (b >= n) break;
    sum += (kv_seq(p.b, p.c.page_shift, p.max_q, b).n_all + kKeys - 1) / kKeys;
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
  const int64_t total = prefix[n] * p.c.n_kv_heads;

  for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
    const int g = (int)(at % p.c.n_kv_heads);
    const int64_t x = at / p.c.n_kv_heads;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (prefix[mid] <= x) lo = mid;
      else hi = mid;
    }
    const KvSeq s = kv_seq(p.b, p.c.page_shift, p.max_q, lo);
    const int key0 = (int)(x - prefix[lo]) * kKeys, ctx = s.n_all - s.n_new;
    const int32_t* table = p.b.page_table + (int64_t)lo * p.b.max_pages;
    const int32_t* perm = p.b.perm ? p.b.perm + s.begin : nullptr;

    // ---- keys to shared memory (bf16; codes of an int8 cache are widened exactly)
    constexpr int kSrc = kI8 ? kD / 16 : kPieces;   // 16-byte pieces of a cached row
#pragma unroll
    for (int c = 0; c < kKeys * kSrc / kThreads; ++c) {
      const int idx = c * kThreads + tid, r = idx / kSrc, pc = idx % kSrc, key = key0 + r;
      int page = -1;
      if (key < s.n_all) page = table[key >> p.c.page_shift];
      const bool ok = (unsigned)page < (unsigned)p.c.n_pages;
      if (!ok && key < s.n_all && p.status) atomicCAS(p.status, MQ_OK, MQ_ERR_INVALID_ARG);
      const int64_t src = ok ? (int64_t)page * p.c.page_stride + (int64_t)g * p.c.head_stride +
                                   (int64_t)(key & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride + pc * 16
                             : 0;
      if (!kI8) {
        cp_async16(kv_smem_u32(ks + r * S::kPitch + pc * 16), ok ? p.c.K + src : p.Q, ok ? 16u : 0u);
      } else {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (ok) v = *reinterpret_cast<const uint4*>(p.c.K + src);
        uint4 a, b;
        i8x4_to_bf16(v.x, a.x, a.y); i8x4_to_bf16(v.y, a.z, a.w);
        i8x4_to_bf16(v.z, b.x, b.y); i8x4_to_bf16(v.w, b.z, b.w);
        *reinterpret_cast<uint4*>(ks + r * S::kPitch + pc * 32) = a;
        *reinterpret_cast<uint4*>(ks + r * S::kPitch + pc * 32 + 16) = b;
      }
    }
    cp_async_commit();

    // ---- query rows that may see any of these keys
    const int n_rows = s.n_new * p.group;
    const int first_tok = perm ? 0 : max(0, key0 - ctx);
    const float scale_log2 = p.scale * 1.4426950408889634f * (kI8 ? p.c.k_scale[g] : 1.0f);
    float sum0 = 0.0f, sum1 = 0.0f;
    const int ka = key0 + warp * 16 + quad, kb = ka + 8;
    uint32_t kf[kSteps][4];
    bool have_k = false;
    for (int r0 = first_tok * p.group; r0 < n_rows; r0 += kRowsQ) {
      __syncthreads();   // the previous block of rows has been read
#pragma unroll
      for (int c = 0; c < kRowsQ * kPieces / kThreads; ++c) {
        const int idx = c * kThreads + tid, r = idx / kPieces, pc = idx % kPieces, row = r0 + r;
        const bool ok = row < n_rows;
        const uint8_t* src = p.Q;
        if (ok) src += (int64_t)(s.begin + row / p.group) * p.ldq + (int64_t)(g * p.group + row % p.group) * (kD * 2) + pc * 16;
        cp_async16(kv_smem_u32(qs + r * S::kPitch + pc * 16), src, ok ? 16u : 0u);
      }
      cp_async_commit();
      if (tid < kRowsQ) {
        const int row = r0 + tid;
        float l = INFINITY;
        int lim = INT_MIN;
        if (row < n_rows) {
          const int tok = row / p.group;
          l = p.lse[(int64_t)(s.begin + tok) * p.n_q_heads + g * p.group + row % p.group] * 1.4426950408889634f;
          if (l == -INFINITY) l = INFINITY;   // a row that sees nothing
          lim = perm ? perm[tok] : ctx + tok + 1;
        }
        row_lse[tid] = l;
        row_lim[tid] = lim;
      }
      cp_async_wait<0>();
      __syncthreads();
      if (!have_k) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
          ldsm_x4(kv_smem_u32(ks + (warp * 16 + (lane & 15)) * S::kPitch + k * 32 + (lane >> 4) * 16), kf[k]);
        have_k = true;
      }
      const int blocks = (min(kRowsQ, n_rows - r0) + 7) / 8;
      // all rows of the step see all keys of the tile?
      const bool masked = key0 + kKeys > (perm ? ctx : ctx + r0 / p.group + 1) || key0 + kKeys > s.n_all;
      for (int nb = 0; nb < blocks; ++nb) {
        float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kSteps; k += 2) {
          uint32_t b[4];
          ldsm_x4(kv_smem_u32(qs + (nb * 8 + (lane & 7)) * S::kPitch + k * 32 + (lane >> 3) * 16), b);
          mma_16816<false>(c, kf[k], b[0], b[1]);
          mma_16816<false>(c, kf[k + 1], b[2], b[3]);
        }
        const int r = nb * 8 + 2 * t4;
        const float2 l = *reinterpret_cast<const float2*>(row_lse + r);
        float e[4] = {kv_exp2(fmaf(c[0], scale_log2, -l.x)), kv_exp2(fmaf(c[1], scale_log2, -l.y)),
                      kv_exp2(fmaf(c[2], scale_log2, -l.x)), kv_exp2(fmaf(c[3], scale_log2, -l.y))};
        if (masked) {
          const int2 lim = *reinterpret_cast<const int2*>(row_lim + r);
          auto sees = [&](int key, int lm) -> bool {
            if (key >= s.n_all || lm == INT_MIN) return false;
            return perm ? key < ctx || perm[key - ctx] <= lm : key < lm;
          };
          if (!sees(ka, lim.x)) e[0] = 0.0f;
          if (!sees(ka, lim.y)) e[1] = 0.0f;
          if (!sees(kb, lim.x)) e[2] = 0.0f;
          if (!sees(kb, lim.y)) e[3] = 0.0f;
        } else if (row_lim[r] == INT_MIN || row_lim[r + 1] == INT_MIN) {   // rows behind the last one
          if (row_lim[r] == INT_MIN) e[0] = e[2] = 0.0f;
          if (row_lim[r + 1] == INT_MIN) e[1] = e[3] = 0.0f;
        }
        sum0 += e[0] + e[1];
        sum1 += e[2] + e[3];
      }
    }
    cp_async_wait<0>();   // (a tile that no row sees loads its keys for nothing)
    sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1); sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2);
    sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1); sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
    if (t4 == 0) {
      const int64_t base = (int64_t)lo * p.seq_stride + (int64_t)g * p.head_stride;
      if (ka < s.n_all) p.W_out[base + ka] = (p.W_in && ka < ctx ? p.W_in[base + ka] : 0.0f) + sum0;
      if (kb < s.n_all) p.W_out[base + kb] = (p.W_in && kb < ctx ? p.W_in[base + kb] : 0.0f) + sum1;
    }
    __syncthreads();   // the keys have been read before the next tile overwrites them
  }
}

template <int kD, bool kI8>
int launch(const WeightParams& p, int64_t most, cudaStream_t st) {
  using S = Smem<kD>;
  const size_t smem = S::kBytes + ((size_t)p.b.n_seq + 1) * sizeof(int64_t);
  static PerDeviceTable<char> attr_set;
  if (!ensure_dynamic_smem(attr_set, kv_weights_kernel<kD, kI8>, S::kBytes + (kMaxKvSeqs + 1) * (int)sizeof(int64_t))) return MQ_ERR_CUDA;
  const int64_t cap = (int64_t)sm_count() * 3;
  const cudaError_t e = launch_pdl(kv_weights_kernel<kD, kI8>, dim3((unsigned)(most < cap ? most : cap)), dim3(kThreads), smem, st, p);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" int mq_kv_weights(const void* Q, int64_t ldq, const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads,
                             float scale, const float* lse, const float* W_in, float* W_out, int64_t w_seq_stride,
                             int64_t w_head_stride, int32_t* status, void* stream) {
  WeightParams p{};
  int rc = check_kv_cache(cache, &p.c);
  if (rc != MQ_OK) return rc;
  if ((rc = check_kv_batch(batch, &p.b)) != MQ_OK) return rc;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads) return MQ_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || !std::isfinite(scale)) return MQ_ERR_INVALID_ARG;
  const int64_t reach = (int64_t)batch->max_pages * cache->page_size;
  if (ldq < (int64_t)n_q_heads * cache->head_dim || w_head_stride < 0 || w_seq_stride < 0) return MQ_ERR_INVALID_ARG;
  if ((int64_t)batch->max_q * (n_q_heads / cache->n_kv_heads) > (1 << 30)) return MQ_ERR_UNSUPPORTED;
  if (batch->n_seq == 0 || reach == 0 || batch->total_q == 0) return MQ_OK;   // (no rows: no weight is added anywhere)
  if (!W_out || !Q || !lse) return MQ_ERR_INVALID_ARG;
  if ((Q && !kv_aligned16(Q)) || ldq % 8) return MQ_ERR_ALIGNMENT;
  p.Q = static_cast<const uint8_t*>(Q);
  p.ldq = ldq * 2;
  p.max_q = batch->max_q;
  p.group = n_q_heads / cache->n_kv_heads;
  p.n_q_heads = n_q_heads;
  p.scale = scale;
  p.lse = lse;
  p.W_in = W_in;
  p.W_out = W_out;
  p.seq_stride = w_seq_stride;
  p.head_stride = w_head_stride;
  p.status = status;
  const int64_t most = (int64_t)batch->n_seq * cache->n_kv_heads * ((reach + kKeys - 1) / kKeys);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool i8 = (cache->flags & MQ_KV_INT8) != 0;
  // (a token's heads have to fit into a row tile of the chunk kernel, and its maps need a page)
  if ((int64_t)batch->max_q * p.group > kFewRows && p.group <= 128 && cache->n_pages > 0)
    return launch_kv_weights_chunk(p, cache->head_dim, i8, most, st);
  if (cache->head_dim == 128) return i8 ? launch<128, true>(p, most, st) : launch<128, false>(p, most, st);
  return i8 ? launch<64, true>(p, most, st) : launch<64, false>(p, most, st);
}
