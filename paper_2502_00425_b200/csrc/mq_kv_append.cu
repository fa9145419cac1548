// Norm of every query and key head, rotary embedding and the store into the paged cache, in one pass:
//   n = x / sqrt(mean(x^2) + eps) * gain;   y = n rotated by pos * base^(-2i / D);   Q_out, K_out, cache <- y, V
// The pass is bound by its bytes (each of q, k, v read once and written once).  A head row of D channels is held by
// D / 8 lanes (16 bytes each), so the sum of squares is a shuffle over those lanes and a row never leaves registers;
// a warp loads all the head rows it will work on before it touches the first one.  The rotation's angle depends on
// (token, pair) only: a lane always holds the same channels, so the sines and cosines are computed once per token and
// warp and serve all of its heads, and the frequencies (doubles) are read once per thread.
// The angle in turns, pos * theta / (2 pi), is formed and reduced in double: in float32 a position of 100,000 would
// leave an angle error of 4e-3.
#include "mq_kv.cuh"

namespace mq {
namespace {

struct AppendParams {
  const uint8_t *Q, *K, *V;
  int64_t ldq, ldk, ldv;     // bytes
  uint8_t *Qo, *Ko;
  int64_t ldqo, ldko;        // bytes
  int T, n_q, n_kv, n_items; // n_items: head-row groups per token
  const float *gain_q, *gain_k;
  float eps;
  const int32_t* pos;
  const int64_t* slots;
  int has_cache;
  KvView c;
  double turns[64];          // theta_i / (2 pi)
};

constexpr int kWarps = 8;

// kD: head dimension; kHalf: pairs (i, i + D/2); kI8: int8 cache; kU: head-row groups a warp loads at once
template <int kD, bool kHalf, bool kI8, int kU>
__global__ void __launch_bounds__(kWarps * 32)
qk_norm_rope_kernel(const __grid_constant__ AppendParams p) {
  constexpr int kLanes = kD / 8;        // lanes per head row
  constexpr int kRows = 32 / kLanes;    // head rows per warp step
  constexpr int kAng = kHalf ? 8 : 4;   // angles a lane needs
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane % kLanes, sel = lane / kLanes;
  double turns[kAng];
#pragma unroll
  for (int e = 0; e < kAng; ++e) turns[e] = p.turns[kHalf ? (8 * sub + e) % (kD / 2) : 4 * sub + e];
  pdl_wait();
  float gq[8], gk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    gq[e] = p.gain_q ? p.gain_q[8 * sub + e] : 1.0f;
    gk[e] = p.gain_k ? p.gain_k[8 * sub + e] : 1.0f;
  }
  const int n_rows = p.n_q + p.n_kv + (p.has_cache ? p.n_kv : 0);   // q heads, k heads, v heads of one token
  const int chunks = (p.n_items + kU - 1) / kU;
  const int64_t n_work = (int64_t)p.T * chunks;
  for (int64_t w = (int64_t)blockIdx.x * kWarps + warp; w < n_work; w += (int64_t)gridDim.x * kWarps) {
    const int t = (int)(w / chunks), c = (int)(w % chunks);
    uint4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int h = (c * kU + u) * kRows + sel;
      x[u] = make_uint4(0u, 0u, 0u, 0u);
      const uint8_t* src = nullptr;
      if (h < p.n_q) src = p.Q + (int64_t)t * p.ldq + (int64_t)h * (kD * 2);
      else if (h < p.n_q + p.n_kv) src = p.K + (int64_t)t * p.ldk + (int64_t)(h - p.n_q) * (kD * 2);
      else if (h < n_rows) src = p.V + (int64_t)t * p.ldv + (int64_t)(h - p.n_q - p.n_kv) * (kD * 2);
      if (src) x[u] = *reinterpret_cast<const uint4*>(src + sub * 16);
    }
    const double pos = (double)p.pos[t];
    int64_t slot = -1;
    if (p.has_cache) slot = p.slots[t];
    float cs[kAng], sn[kAng];
#pragma unroll
    for (int e = 0; e < kAng; ++e) {
      const double rev = pos * turns[e];
      sincospif(2.0f * (float)(rev - rint(rev)), &sn[e], &cs[e]);
    }
    const int64_t page = slot >> p.c.page_shift;
    const bool stored = p.has_cache && slot >= 0 && page < p.c.n_pages;
    const int64_t row_off = stored ? page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride : 0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int h = (c * kU + u) * kRows + sel;
      const uint32_t xw[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[2 * e] = kv_bf16_lo(xw[e]); v[2 * e + 1] = kv_bf16_hi(xw[e]); }
      const bool is_q = h < p.n_q, is_k = !is_q && h < p.n_q + p.n_kv;
      const bool norm = is_q ? p.gain_q != nullptr : is_k && p.gain_k != nullptr;
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (norm) {
        const float r = rsqrtf(ss * (1.0f / kD) + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * r * (is_q ? gq[e] : gk[e]);
      }
      float y[8];
      if (kHalf) {
        const bool second = sub >= kLanes / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float mate = __shfl_xor_sync(0xffffffffu, v[e], kLanes / 2);
          y[e] = second ? fmaf(mate, sn[e % kAng], v[e] * cs[e % kAng]) : fmaf(-mate, sn[e % kAng], v[e] * cs[e % kAng]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[2 * e] = fmaf(-v[2 * e + 1], sn[e], v[2 * e] * cs[e]);
          y[2 * e + 1] = fmaf(v[2 * e + 1], cs[e], v[2 * e] * sn[e]);
        }
      }
      if (!is_q && !is_k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = v[e];
      }
      const uint4 o = make_uint4(kv_pack_bf16(y[0], y[1]), kv_pack_bf16(y[2], y[3]), kv_pack_bf16(y[4], y[5]), kv_pack_bf16(y[6], y[7]));
      if (is_q) {
        *reinterpret_cast<uint4*>(p.Qo + (int64_t)t * p.ldqo + (int64_t)h * (kD * 2) + sub * 16) = o;
      } else if (h < n_rows) {
        const int g = is_k ? h - p.n_q : h - p.n_q - p.n_kv;
        if (is_k && p.Ko) *reinterpret_cast<uint4*>(p.Ko + (int64_t)t * p.ldko + (int64_t)g * (kD * 2) + sub * 16) = o;
        if (stored) {
          uint8_t* dst = const_cast<uint8_t*>(is_k ? p.c.K : p.c.V) + row_off + (int64_t)g * p.c.head_stride;
          if (kI8) {
            const float inv = 1.0f / (is_k ? p.c.k_scale[g] : p.c.v_scale[g]);
            uint32_t q[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int code = max(-128, min(127, __float2int_rn(y[e] * inv)));
              q[e >> 2] |= (uint32_t)(code & 255) << (8 * (e & 3));
            }
            *reinterpret_cast<uint2*>(dst + sub * 8) = make_uint2(q[0], q[1]);
          } else {
            *reinterpret_cast<uint4*>(dst + sub * 16) = o;
          }
        }
      }
    }
  }
}

template <int kD, bool kHalf, bool kI8>
int launch(AppendParams& p, cudaStream_t st) {
  const int rows = p.n_q + p.n_kv * (p.has_cache ? 2 : 1);
  constexpr int per = 32 / (kD / 8);
  p.n_items = (rows + per - 1) / per;
  const int sms = sm_count();
  // few tokens: one head-row group per warp, so that the call is one latency long; many: six loads in flight per lane
  const bool wide = (int64_t)p.T * p.n_items > (int64_t)sms * 64;
  const int64_t work = (int64_t)p.T * (wide ? (p.n_items + 5) / 6 : p.n_items);
  const int64_t blocks = (work + kWarps - 1) / kWarps;
  const unsigned grid = (unsigned)(blocks < (int64_t)sms * 8 ? blocks : (int64_t)sms * 8);
  const cudaError_t e = wide ? launch_pdl(qk_norm_rope_kernel<kD, kHalf, kI8, 6>, dim3(grid), dim3(kWarps * 32), 0, st, p)
                             : launch_pdl(qk_norm_rope_kernel<kD, kHalf, kI8, 1>, dim3(grid), dim3(kWarps * 32), 0, st, p);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" int mq_qk_norm_rope(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                               int32_t T, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const float* gain_q,
                               const float* gain_k, float eps, const int32_t* pos, float base, uint32_t flags, void* Q_out,
                               int64_t ldqo, void* K_out, int64_t ldko, const mq_kv_cache* cache, const int64_t* slots,
                               void* stream) {
  if (T < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || head_dim <= 0 || (flags & ~MQ_ROPE_HALF)) return MQ_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !std::isfinite(eps) || !(base > 1.0f) || !std::isfinite(base)) return MQ_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return MQ_ERR_UNSUPPORTED;
  if (n_q_heads > 65536 || n_kv_heads > 65536) return MQ_ERR_UNSUPPORTED;
  AppendParams p{};
  if (cache) {
    const int rc = check_kv_cache(cache, &p.c);
    if (rc != MQ_OK) return rc;
    if (cache->head_dim != head_dim || cache->n_kv_heads != n_kv_heads) return MQ_ERR_INVALID_ARG;
  }
  const int64_t wq = (int64_t)n_q_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
  if (ldq < wq || ldk < wk || ldqo < wq || (K_out && ldko < wk) || (cache && ldv < wk)) return MQ_ERR_INVALID_ARG;
  if (T == 0) return MQ_OK;
  if (!Q || !K || !pos || !Q_out || (!cache && !K_out) || (cache && (!V || !slots))) return MQ_ERR_INVALID_ARG;
  if (!kv_aligned16(Q) || !kv_aligned16(K) || !kv_aligned16(Q_out) || (K_out && !kv_aligned16(K_out)) || (cache && !kv_aligned16(V)) ||
      (gain_q && !kv_aligned16(gain_q)) || (gain_k && !kv_aligned16(gain_k)) || ldq % 8 || ldk % 8 || ldqo % 8 ||
      (K_out && ldko % 8) || (cache && ldv % 8))
    return MQ_ERR_ALIGNMENT;
  p.Q = static_cast<const uint8_t*>(Q); p.K = static_cast<const uint8_t*>(K); p.V = static_cast<const uint8_t*>(V);
  p.ldq = ldq * 2; p.ldk = ldk * 2; p.ldv = ldv * 2;
  p.Qo = static_cast<uint8_t*>(Q_out); p.Ko = static_cast<uint8_t*>(K_out);
  p.ldqo = ldqo * 2; p.ldko = ldko * 2;
  p.T = T; p.n_q = n_q_heads; p.n_kv = n_kv_heads;
  p.gain_q = gain_q; p.gain_k = gain_k; p.eps = eps; p.pos = pos; p.slots = slots;
  p.has_cache = cache != nullptr;
  // powers of one ratio, in long double: 64 roundings of 2^-64 (one pow instead of 64, which took longer than the launch)
  const long double ratio = powl((long double)base, -2.0L / head_dim);
  long double turn = 1.0L / 6.283185307179586476925286766559L;
  for (int i = 0; i < head_dim / 2; ++i, turn *= ratio) p.turns[i] = (double)turn;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool half = flags & MQ_ROPE_HALF, i8 = cache && (cache->flags & MQ_KV_INT8);
  if (head_dim == 128) {
    if (half) return i8 ? launch<128, true, true>(p, st) : launch<128, true, false>(p, st);
    return i8 ? launch<128, false, true>(p, st) : launch<128, false, false>(p, st);
  }
  if (half) return i8 ? launch<64, true, true>(p, st) : launch<64, true, false>(p, st);
  return i8 ? launch<64, false, true>(p, st) : launch<64, false, false>(p, st);
}
