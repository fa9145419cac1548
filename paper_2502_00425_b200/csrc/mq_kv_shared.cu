// Attention of sequences that share a prefix over a paged cache: two lines of work with the kernels of mq_kv_attn.cu and
// mq_kv_chunk.cu, and a kernel that joins what they leave.
//
//   O = (e^(m1 - m) o1 + e^(m2 - m) o2) / (e^(m1 - m) l1 + e^(m2 - m) l2),  m = max(m1, m2)
// with (m, l, o) the exponents' reference, the sum and the unnormalised output over the shared keys and over a sequence's own.
// The shared line has all tokens of a group of sequences as the rows of one list of keys, so a shared key is read once per 256 rows and meets the
// 128-row tensor-memory kernel even where every sequence has one new token; the own line is an ordinary step over shorter lists.
// 128 sequences of one new token over 32768 shared keys (32 / 8 heads of 128, bf16): 134 us, of which the prefix line takes 75 (0.9 PFLOP/s: products
// and exponentials in turn), the own line 57 (5.5 TB/s), the join 8; every sequence by itself 1265.  32 over 3360 keys (28 / 4 heads): 27 us, the latency of the
// two lines and the join, as long as it takes without sharing, where the repeated reads come out of L2.
#include <cmath>

#include "mq_kv_sched.cuh"

namespace mq {
namespace {

struct JoinArgs {
  KvWhole line[2];         // kPrefix, kOwn
  KvParts parts[2];
  int pitch[2], workers[2];
  KvOutArgs out;
};

// Joins what the two lines left of a row: first over the shared keys, then over its own, each in the order of the keys.  kW warps
// share a row and take every kW-th piece.
template <int kD, int kW>
__global__ void __launch_bounds__(256) kv_join_kernel(const __grid_constant__ JoinArgs p) {
  constexpr int kPer = kD / 32, kRows = 8 / kW;
  __shared__ float part[kRows][kW][kD + 2];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rr = warp / kW, pw = warp % kW;
  const int64_t row = (int64_t)blockIdx.x * kRows + rr;
  KvRowRef ref[2] = {{0, -1, 0, 0}, {0, -1, 0, 0}};
  KvRowRef shared_ref = {0, -1, 0, 0};
  if (row < p.line[1].n_rows) {
    ref[1] = p.line[1].ref[row];
    shared_ref = p.line[0].ref[row];   // (asked for along; it says something only if the other one says so)
  }
  const bool live = ref[1].n_parts >= 0;
  if (live && ref[1].more) ref[0] = shared_ref;
  float m = -INFINITY, l = 0.0f, x[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const KvRowRef& f = ref[k];
    // (a line that gave up may have left anything in its references; the status says so)
    if (f.n_parts < 0 || f.worker < 0 || f.row < 0 || f.row >= p.pitch[k] || (int64_t)f.worker + f.n_parts > p.workers[k]) continue;
    const int n = f.n_parts == 0 ? 1 : f.n_parts;
    constexpr int kBatch = 4;
    for (int i0 = pw; i0 < n; i0 += kBatch * kW) {
      float2 ml[kBatch];
      float v[kBatch][kPer];
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        const int i = i0 + c * kW;
        ml[c] = make_float2(-INFINITY, 0.0f);
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[c][e] = 0.0f;
        if (i < n) {
          const int64_t at = f.n_parts == 0 ? row : (int64_t)(i == 0 ? 2 * f.worker + 1 : 2 * (f.worker + i)) * p.pitch[k] + f.row;
          ml[c] = f.n_parts == 0 ? p.line[k].ml[at] : p.parts[k].ml[at];
          const float* src = (f.n_parts == 0 ? p.line[k].o : p.parts[k].o) + at * kD + lane * kPer;
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
      const float back = m == -INFINITY ? 0.0f : kv_exp2(m - top);
      l *= back;
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] *= back;
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        // (a reference of -inf: nothing but zeros, or scores that are all NaN, whose sum says so and is kept)
        const float w = ml[c].x == -INFINITY ? 0.0f : kv_exp2(ml[c].x - top);
        l = fmaf(w, ml[c].y, l);
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = fmaf(w, v[c][e], x[e]);
      }
      m = top;
    }
  }
  if (kW > 1) {
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
    for (int k = 1; k < kW; ++k) m = fmaxf(m, part[rr][k][kD]);
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < kW; ++k) {
      const float mk = part[rr][k][kD];
      const float w = mk == -INFINITY ? 0.0f : kv_exp2(mk - m);
      l = fmaf(w, part[rr][k][kD + 1], l);
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] = fmaf(w, part[rr][k][lane * kPer + e], x[e]);
    }
  }
  if (!live) return;
  const int64_t tok = row / p.out.n_q_heads;
  const int head = (int)(row - tok * p.out.n_q_heads);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  __nv_bfloat16* dst = p.out.O + tok * p.out.ldo + (int64_t)head * kD + lane * kPer;
  if (kPer == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(kv_pack_bf16(x[0] * inv, x[1] * inv), kv_pack_bf16(x[2 % kPer] * inv, x[3 % kPer] * inv));
  else
    *reinterpret_cast<uint32_t*>(dst) = kv_pack_bf16(x[0] * inv, x[1] * inv);
  if (lane == 0 && p.out.lse) p.out.lse[row] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <int kD>
cudaError_t launch_shared_join(const JoinArgs& j, cudaStream_t st) {
  // few rows have their keys spread over many workers: four warps to a row (896 rows of 8 to 14 pieces: the call 27.3 us, 29.2 with one)
  if (j.line[1].n_rows <= 2048) return launch_pdl(kv_join_kernel<kD, 4>, dim3((unsigned)((j.line[1].n_rows + 1) / 2)), dim3(256), 0, st, j);
  return launch_pdl(kv_join_kernel<kD, 1>, dim3((unsigned)((j.line[1].n_rows + 7) / 8)), dim3(256), 0, st, j);
}

struct SharedPlan {
  KvPlan line[2];            // kPrefix, kOwn
  size_t parts[2], ref, ml, o, bytes;
};
SharedPlan shared_plan(const mq_kv_batch* b, const mq_kv_cache* c, int n_q_heads) {
  SharedPlan s{};
  const int group = n_q_heads / c->n_kv_heads;
  // (a group is two sequences at least)
  s.line[0] = kv_plan_attention(b, c, group, b->n_seq / 2, b->total_q);
  s.line[1] = kv_plan_attention(b, c, group, b->n_seq, b->max_q);
  const size_t rows = (size_t)b->total_q * n_q_heads;
  for (int k = 0; k < 2; ++k) s.parts[k] = align_up(kv_parts_bytes(s.line[k].workers, s.line[k].pitch, c->head_dim), 256);
  s.ref = align_up(rows * sizeof(KvRowRef), 256);
  s.ml = align_up(rows * sizeof(float2), 256);
  s.o = align_up(rows * c->head_dim * sizeof(float), 256);
  s.bytes = kStatusBytes + s.parts[0] + s.parts[1] + 2 * (s.ref + s.ml + s.o);
  return s;
}

int check_shared(const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads, KvBatchView* bv, KvView* cv) {
  const int rc = check_kv_attention(batch, cache, n_q_heads, bv, cv);
  if (rc != MQ_OK) return rc;
  if (batch->n_seq > kMaxSharedSeqs) return MQ_ERR_UNSUPPORTED;
  // rows of a group (all tokens x heads of the group) are int32, as the join's blocks are
  if ((int64_t)batch->total_q * n_q_heads > (1 << 30)) return MQ_ERR_UNSUPPORTED;
  return MQ_OK;
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" size_t mq_kv_attention_shared_workspace_bytes(const mq_kv_batch* batch, const mq_kv_cache* cache, int32_t n_q_heads) {
  KvBatchView bv;
  KvView cv;
  if (check_shared(batch, cache, n_q_heads, &bv, &cv) != MQ_OK) return 0;
  return shared_plan(batch, cache, n_q_heads).bytes;
}

extern "C" int mq_kv_attention_shared(const void* Q, int64_t ldq, const mq_kv_batch* batch, const int32_t* leader, const int32_t* shared_len,
                                      const mq_kv_cache* cache, int32_t n_q_heads, float scale, void* O, int64_t ldo, float* lse, void* ws,
                                      size_t ws_bytes, void* stream) {
  KvAttnArgs a{};
  const int rc = check_shared(batch, cache, n_q_heads, &a.sched.b, &a.cache);
  if (rc != MQ_OK) return rc;
  if (!(scale > 0.0f) || !std::isfinite(scale)) return MQ_ERR_INVALID_ARG;
  const int64_t width = (int64_t)n_q_heads * cache->head_dim;
  if (ldq < width || ldo < width) return MQ_ERR_INVALID_ARG;
  if (batch->n_seq == 0 || batch->total_q == 0 || batch->max_q == 0) return MQ_OK;
  if (!Q || !O || !ws || !leader || !shared_len) return MQ_ERR_INVALID_ARG;
  if (!kv_aligned16(Q) || !kv_aligned16(O) || ldq % 8 || ldo % 8 || (reinterpret_cast<uintptr_t>(ws) & 255u)) return MQ_ERR_ALIGNMENT;
  const SharedPlan s = shared_plan(batch, cache, n_q_heads);
  if (ws_bytes < s.bytes) return MQ_ERR_WORKSPACE;
  const int group = n_q_heads / cache->n_kv_heads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.Q = static_cast<const uint8_t*>(Q);
  a.ldq = ldq * 2;
  a.sched.leader = leader;
  a.sched.shared_len = shared_len;
  a.out.O = static_cast<__nv_bfloat16*>(O);
  a.out.ldo = ldo;
  a.out.lse = lse;
  a.out.n_q_heads = n_q_heads;
  a.scale = scale;
  a.status = static_cast<int32_t*>(ws);
  JoinArgs j{};
  j.out = a.out;
  uint8_t* at = static_cast<uint8_t*>(ws) + kStatusBytes;
  for (int k = 0; k < 2; ++k) {
    j.parts[k] = kv_parts(at, s.line[k].workers, s.line[k].pitch);
    at += s.parts[k];
    j.line[k].ref = reinterpret_cast<KvRowRef*>(at);
    at += s.ref;
    j.line[k].ml = reinterpret_cast<float2*>(at);
    at += s.ml;
    j.line[k].o = reinterpret_cast<float*>(at);
    at += s.o;
    j.line[k].n_rows = (int64_t)batch->total_q * n_q_heads;
    j.pitch[k] = s.line[k].pitch;
    j.workers[k] = s.line[k].workers;
  }
  j.line[0].clear = j.line[1].ref;
  for (int k = 0; k < 2; ++k) {
    kv_set_plan(&a, s.line[k], cache, batch->max_q, group);
    // short prefixes are spread further than an ordinary chunk's keys: 32 tokens over 3328 keys 31.4 us with the chunks' least share of a
    // worker (4 tiles with the fixed cost), 30.3 with 2, 34.9 with 1
    if (k == 0 && s.line[0].chunk) a.sched.min_len = 2;
    a.parts = j.parts[k];
    a.whole = j.line[k];
    const int e = launch_kv_lines(a, s.line[k], k ? kOwn : kPrefix, cache->head_dim, (cache->flags & MQ_KV_INT8) != 0, st);
    if (e != MQ_OK) return e;
  }
  const cudaError_t e = cache->head_dim == 128 ? launch_shared_join<128>(j, st) : launch_shared_join<64>(j, st);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(cudaGetLastError());
}
