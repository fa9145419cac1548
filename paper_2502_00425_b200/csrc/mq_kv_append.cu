// Norm of every query and key head, rotary embedding and the store into the paged cache, in one pass:
//   n = x / sqrt(mean(x^2) + eps) * gain;   y = n rotated by pos * base^(-2i / D);   Q_out, K_out, cache <- y, V
// The pass is bound by its bytes (each of q, k, v read once and written once).  A head row of D channels is held by
// D / 8 lanes, so the sum of squares is a shuffle over those lanes and a row never leaves registers; a lane's 8 channels
// are four pairs: 16 contiguous bytes, or for pairs (i, i + D/2) two runs of 8 bytes, so that no pair crosses lanes.
// A warp works on (a part of) a token: it loads several head rows before it touches the first one.  The rotation's angle
// depends on (token, pair) only, and a lane always holds the same pairs: four sines and cosines per token serve all of
// its heads (they cost as much as two head rows), and the frequencies (doubles) are read once per thread.
// The angle in turns, pos * theta / (2 pi), is formed and reduced in double: in float32 a position of 100,000 would
// leave an angle error of 4e-3.
// 9728 tokens of 32 + 8 heads of 128, 239 MB: 53 us, 4.5 TB/s (68 % of a plain copy).  39 M warp instructions (sums, conversions,
// rotation) are 35 us of issue by themselves, as long as the bytes take; issue is busy for 68 % of the cycles in which an SM
// has work, the rest are fixed latencies and the shuffles' and conversions' results (7 warps to a scheduler), and 11 % of the
// time an SM has none (start, last round).  Into an int8 cache: 6 us more.  32 tokens: 3.4 us.
#include "mq_kv.cuh"

namespace mq {
namespace {

struct AppendParams {
  const uint8_t *Q, *K, *V;
  int64_t ldq, ldk, ldv;     // bytes
  uint8_t *Qo, *Ko;
  int64_t ldqo, ldko;        // bytes
  int T, n_q, n_kv;
  int n_steps;               // steps of 32 lanes per token
  int chunks, per_chunk;     // parts that a token's steps are cut into, and the steps of a part
  const float *gain_q, *gain_k;
  float eps;
  const int32_t* pos;
  const int64_t* slots;
  int has_cache;
  KvView c;
  double turns[64];          // theta_i / (2 pi)
};

constexpr int kWarps = 8;

// kD: head dimension; kHalf: pairs (i, i + D/2); kI8: int8 cache; kU: steps of 32 lanes that a warp loads at once
template <int kD, bool kHalf, bool kI8, int kU>
__global__ void __launch_bounds__(kWarps * 32, kU > 1 ? 4 : 2)
qk_norm_rope_kernel(const __grid_constant__ AppendParams p) {
  constexpr int kLanes = kD / 8;        // lanes per head row
  constexpr int kRows = 32 / kLanes;    // head rows per step
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane % kLanes, sel = lane / kLanes;
  // byte offsets of a lane's two runs of four channels
  const int off0 = kHalf ? sub * 8 : sub * 16, off1 = kHalf ? kD + sub * 8 : sub * 16 + 8;
  double turns[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) turns[e] = p.turns[4 * sub + e];
  pdl_wait();
  const int n_rows = p.n_q + p.n_kv + (p.has_cache ? p.n_kv : 0);   // q heads, k heads, v heads of one token
  const int64_t n_work = (int64_t)p.T * p.chunks;
  for (int64_t w = (int64_t)blockIdx.x * kWarps + warp; w < n_work; w += (int64_t)gridDim.x * kWarps) {
    const int t = p.chunks == 1 ? (int)w : (int)(w / p.chunks), part = p.chunks == 1 ? 0 : (int)(w - (int64_t)t * p.chunks);
    const uint8_t *q_row = p.Q + (int64_t)t * p.ldq, *k_row = p.K + (int64_t)t * p.ldk, *v_row = p.V + (int64_t)t * p.ldv;
    const int s_end = min(p.n_steps, (part + 1) * p.per_chunk);
    float cs[4], sn[4];
    bool stored = false;
    int64_t row_off = 0;
    for (int s0 = part * p.per_chunk; s0 < s_end; s0 += kU) {
      uint2 x[kU][2];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int h = (s0 + u) * kRows + sel;
        x[u][0] = x[u][1] = make_uint2(0u, 0u);
        if (s0 + u < s_end && h < n_rows) {
          const uint8_t* src = h < p.n_q ? q_row + h * (kD * 2)
                               : h < p.n_q + p.n_kv ? k_row + (h - p.n_q) * (kD * 2) : v_row + (h - p.n_q - p.n_kv) * (kD * 2);
          if (kHalf) {
            x[u][0] = *reinterpret_cast<const uint2*>(src + off0);
            x[u][1] = *reinterpret_cast<const uint2*>(src + off1);
          } else {
            const uint4 y = *reinterpret_cast<const uint4*>(src + off0);
            x[u][0] = make_uint2(y.x, y.y);
            x[u][1] = make_uint2(y.z, y.w);
          }
        }
      }
      if (s0 == part * p.per_chunk) {   // (while the first loads are on their way)
        const double pos = (double)p.pos[t];
        const int64_t slot = p.has_cache ? p.slots[t] : -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double rev = pos * turns[e];
          sincospif(2.0f * (float)(rev - rint(rev)), &sn[e], &cs[e]);
        }
        const int64_t page = slot >> p.c.page_shift;
        stored = slot >= 0 && page < p.c.n_pages;
        row_off = stored ? page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride : 0;
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int h = (s0 + u) * kRows + sel;
        if (s0 + u >= s_end) continue;                       // (the same for all lanes)
        const bool is_q = h < p.n_q, is_k = !is_q && h < p.n_q + p.n_kv;
        float a[4], b[4];   // the pairs
        if (kHalf) {
          a[0] = kv_bf16_lo(x[u][0].x); a[1] = kv_bf16_hi(x[u][0].x); a[2] = kv_bf16_lo(x[u][0].y); a[3] = kv_bf16_hi(x[u][0].y);
          b[0] = kv_bf16_lo(x[u][1].x); b[1] = kv_bf16_hi(x[u][1].x); b[2] = kv_bf16_lo(x[u][1].y); b[3] = kv_bf16_hi(x[u][1].y);
        } else {
          a[0] = kv_bf16_lo(x[u][0].x); b[0] = kv_bf16_hi(x[u][0].x); a[1] = kv_bf16_lo(x[u][0].y); b[1] = kv_bf16_hi(x[u][0].y);
          a[2] = kv_bf16_lo(x[u][1].x); b[2] = kv_bf16_hi(x[u][1].x); a[3] = kv_bf16_lo(x[u][1].y); b[3] = kv_bf16_hi(x[u][1].y);
        }
        const float* gain = is_q ? p.gain_q : is_k ? p.gain_k : nullptr;
        if (p.gain_q || p.gain_k) {                          // (the same for all lanes)
          float ss = 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          if (gain) {
            const float r = rsqrtf(ss * (1.0f / kD) + p.eps);
            const float4 g0 = *reinterpret_cast<const float4*>(gain + off0 / 2), g1 = *reinterpret_cast<const float4*>(gain + off1 / 2);
            const float ga[4] = {g0.x, kHalf ? g0.y : g0.z, kHalf ? g0.z : g1.x, kHalf ? g0.w : g1.z};
            const float gb[4] = {kHalf ? g1.x : g0.y, kHalf ? g1.y : g0.w, kHalf ? g1.z : g1.y, g1.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { a[e] *= r * ga[e]; b[e] *= r * gb[e]; }
          }
        }
        if (is_q || is_k) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = fmaf(-b[e], sn[e], a[e] * cs[e]);
            b[e] = fmaf(b[e], cs[e], a[e] * sn[e]);
            a[e] = y;
          }
        }
        if (h >= n_rows) continue;
        const uint2 o0 = kHalf ? make_uint2(kv_pack_bf16(a[0], a[1]), kv_pack_bf16(a[2], a[3])) : make_uint2(kv_pack_bf16(a[0], b[0]), kv_pack_bf16(a[1], b[1]));
        const uint2 o1 = kHalf ? make_uint2(kv_pack_bf16(b[0], b[1]), kv_pack_bf16(b[2], b[3])) : make_uint2(kv_pack_bf16(a[2], b[2]), kv_pack_bf16(a[3], b[3]));
        auto put = [&](uint8_t* dst) {
          if (kHalf) {
            *reinterpret_cast<uint2*>(dst + off0) = o0;
            *reinterpret_cast<uint2*>(dst + off1) = o1;
          } else {
            *reinterpret_cast<uint4*>(dst + off0) = make_uint4(o0.x, o0.y, o1.x, o1.y);
          }
        };
        if (is_q) {
          put(p.Qo + (int64_t)t * p.ldqo + h * (kD * 2));
        } else {
          const int g = is_k ? h - p.n_q : h - p.n_q - p.n_kv;
          if (is_k && p.Ko) put(p.Ko + (int64_t)t * p.ldko + g * (kD * 2));
          if (stored) {
            uint8_t* dst = const_cast<uint8_t*>(is_k ? p.c.K : p.c.V) + row_off + (int64_t)g * p.c.head_stride;
            if (kI8) {
              const float inv = 1.0f / (is_k ? p.c.k_scale[g] : p.c.v_scale[g]);
              auto code = [&](float y) { return (uint32_t)max(-128, min(127, __float2int_rn(y * inv))) & 255u; };
              uint32_t ca[4], cb[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) { ca[e] = code(a[e]); cb[e] = code(b[e]); }
              if (kHalf) {
                *reinterpret_cast<uint32_t*>(dst + off0 / 2) = ca[0] | ca[1] << 8 | ca[2] << 16 | ca[3] << 24;
                *reinterpret_cast<uint32_t*>(dst + off1 / 2) = cb[0] | cb[1] << 8 | cb[2] << 16 | cb[3] << 24;
              } else {
                *reinterpret_cast<uint2*>(dst + off0 / 2) = make_uint2(ca[0] | cb[0] << 8 | ca[1] << 16 | cb[1] << 24, ca[2] | cb[2] << 8 | ca[3] << 16 | cb[3] << 24);
              }
            } else {
              put(dst);
            }
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
  p.n_steps = (rows + per - 1) / per;
  const int sms = sm_count();
  // few tokens: one step per warp, so that the call is one latency long; many: a warp takes a token, or half of one where
  // that leaves the last warps less to wait for, with four steps in flight.  28 + 4 heads of 128, one step / four steps in
  // us: 2.9 / 5.9 for 1 token, 4.5 / 6.6 for 128, 6.7 / 6.8 for 256 (18 steps each), 10.1 / 7.4 for 512, 59 / 22 for 4096.
  const bool wide = (int64_t)p.T * p.n_steps > (int64_t)sms * 32;
  p.chunks = !wide ? p.n_steps : p.n_steps > 8 ? 2 : 1;
  p.per_chunk = (p.n_steps + p.chunks - 1) / p.chunks;
  const int64_t blocks = ((int64_t)p.T * p.chunks + kWarps - 1) / kWarps, most = (int64_t)sms * 4;
  const unsigned grid = (unsigned)(!wide || blocks < most ? blocks : most);
  const cudaError_t e = wide ? launch_pdl(qk_norm_rope_kernel<kD, kHalf, kI8, 4>, dim3(grid), dim3(kWarps * 32), 0, st, p)
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
    if (cache->head_dim != head_dim || cache->n_kv_heads != n_kv_heads || !kv_rows_apart(cache)) return MQ_ERR_INVALID_ARG;
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
