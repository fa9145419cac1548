// Shared pieces of the key/value-cache kernels (mq_kv_*.cu): the device view of a paged cache, argument checks of
// the two descriptors, and the few warp-level tensor-core instructions (mma.sync, ldmatrix, movmatrix) that the
// kernels with few query rows use.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>
#include <cmath>

#include "mq_common.cuh"

namespace mq {

// Device view of a paged cache.  All strides in BYTES; a row (one key of one head) is head_dim contiguous elements.
struct KvView {
  const uint8_t* K;
  const uint8_t* V;
  int64_t page_stride, head_stride, slot_stride;
  int n_pages, page_shift, n_kv_heads;
  const float* k_scale;   // int8 cache: one static scale per key/value head, else nullptr
  const float* v_scale;
};

// Device view of a ragged batch of new tokens over the cache.
struct KvBatchView {
  int n_seq, total_q, max_pages;
  const int32_t* cu_q;
  const int32_t* kv_len;
  const int32_t* page_table;
  const int32_t* perm;
};

inline bool kv_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_kv_cache(const mq_kv_cache* c, KvView* out) {
  if (!c) return MQ_ERR_INVALID_ARG;
  if (c->flags & ~MQ_KV_INT8) return MQ_ERR_INVALID_ARG;
  const bool i8 = (c->flags & MQ_KV_INT8) != 0;
  if (c->n_pages < 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->page_size <= 0) return MQ_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return MQ_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return MQ_ERR_UNSUPPORTED;
  if (c->n_pages > 0 && (!c->K || !c->V)) return MQ_ERR_INVALID_ARG;
  if (i8 != (c->k_scale != nullptr) || i8 != (c->v_scale != nullptr)) return MQ_ERR_INVALID_ARG;
  const int64_t es = i8 ? 1 : 2;
  // a row is contiguous, no stride is shorter than a row, and every row starts on a 16-byte boundary
  if (c->slot_stride < c->head_dim || c->head_stride < c->head_dim || c->page_stride < c->head_dim) return MQ_ERR_INVALID_ARG;
  const int64_t lim = (int64_t)1 << 38;
  if (c->slot_stride > lim || c->head_stride > lim || c->page_stride > lim) return MQ_ERR_UNSUPPORTED;
  if (!kv_aligned16(c->K) || !kv_aligned16(c->V) || (c->slot_stride * es) % 16 || (c->head_stride * es) % 16 ||
      (c->page_stride * es) % 16)
    return MQ_ERR_ALIGNMENT;
  out->K = static_cast<const uint8_t*>(c->K);
  out->V = static_cast<const uint8_t*>(c->V);
  out->page_stride = c->page_stride * es;
  out->head_stride = c->head_stride * es;
  out->slot_stride = c->slot_stride * es;
  out->n_pages = c->n_pages;
  out->n_kv_heads = c->n_kv_heads;
  out->page_shift = 31 - __builtin_clz((unsigned)c->page_size);
  out->k_scale = c->k_scale;
  out->v_scale = c->v_scale;
  return MQ_OK;
}

// Whether no two of the blocks of `extent` elements that `n` strides and counts span share memory: in the order of their strides,
// each must step over all that the smaller ones reach.
inline bool kv_apart(int64_t extent, int n, const int64_t* stride, const int64_t* count) {
  unsigned done = 0;
  __int128 reach = extent;
  for (int i = 0; i < n; ++i) {
    int k = -1;
    for (int j = 0; j < n; ++j)
      if (!(done >> j & 1u) && (k < 0 || stride[j] < stride[k])) k = j;
    done |= 1u << k;
    if (count[k] <= 1) continue;
    if (stride[k] < reach) return false;
    reach += (__int128)(count[k] - 1) * stride[k];
  }
  return true;
}
// The rows of a cache that is written to (reading shared rows is harmless).
inline bool kv_rows_apart(const mq_kv_cache* c) {
  const int64_t stride[3] = {c->slot_stride, c->head_stride, c->page_stride}, count[3] = {c->page_size, c->n_kv_heads, c->n_pages};
  return kv_apart(c->head_dim, 3, stride, count);
}

constexpr int kMaxKvSeqs = 2048;   // sequences of one call: every CTA keeps a prefix over them in shared memory

inline int check_kv_batch(const mq_kv_batch* b, KvBatchView* out) {
  if (!b) return MQ_ERR_INVALID_ARG;
  if (b->n_seq < 0 || b->total_q < 0 || b->max_q < 0 || b->max_pages < 0 || b->max_q > b->total_q) return MQ_ERR_INVALID_ARG;
  if (b->n_seq > kMaxKvSeqs) return MQ_ERR_UNSUPPORTED;
  // lengths and positions are int32: 2^31 keys of a sequence are out of range whatever the page size (<= 256)
  if (b->max_pages > (1 << 22)) return MQ_ERR_UNSUPPORTED;
  if (b->n_seq > 0 && (!b->cu_q || !b->kv_len)) return MQ_ERR_INVALID_ARG;
  if (b->n_seq > 0 && b->max_pages > 0 && !b->page_table) return MQ_ERR_INVALID_ARG;
  out->n_seq = b->n_seq;
  out->total_q = b->total_q;
  out->max_pages = b->max_pages;
  out->cu_q = b->cu_q;
  out->kv_len = b->kv_len;
  out->page_table = b->page_table;
  out->perm = b->perm;
  return MQ_OK;
}

// Rows [begin, begin + len) of the new tokens of sequence b, kept inside [0, total_q) whatever cu_q holds, and its
// number of keys, kept inside the page table's reach.
struct KvSeq {
  int begin, n_new, n_all;
};
__device__ __forceinline__ KvSeq kv_seq(const KvBatchView& v, int page_shift, int max_q, int b) {
  KvSeq s;
  const int lo = min(max(v.cu_q[b], 0), v.total_q), hi = min(max(v.cu_q[b + 1], lo), v.total_q);
  s.begin = lo;
  s.n_new = min(hi - lo, max_q);
  const int64_t reach = (int64_t)v.max_pages << page_shift;
  s.n_all = (int)min((int64_t)max(v.kv_len[b], 0), reach);
  return s;
}

// Division of 0 <= n < 2^31 by a divisor known on the host: n * m >> 31 + l with l = ceil(log2 d), m = ceil(2^(31 + l) / d)
// (m < 2^32, and the quotient is exact for n < 2^31: Granlund and Montgomery, "Division by invariant integers using
// multiplication", 1994).  A runtime division is some 40 dependent instructions, which
// counts in kernels that last a few microseconds.
struct FastDiv {
  uint32_t m;
  int32_t l, d;
};
inline FastDiv fast_div(int d) {
  FastDiv f;
  f.d = d;
  f.l = 0;
  while (((int64_t)1 << f.l) < d) ++f.l;
  f.m = (uint32_t)((((uint64_t)1 << (31 + f.l)) + d - 1) / d);
  return f;
}
__device__ __forceinline__ int operator/(int n, const FastDiv& f) { return (int)(((uint64_t)(uint32_t)n * f.m) >> (31 + f.l)); }

// ---- instructions ---------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t kv_smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// The transpose of an 8 x 8 matrix of 16-bit values held as two neighbouring columns per lane
__device__ __forceinline__ uint32_t mat_transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// D (16 x 8, float32) += A (16 x 16) B (16 x 8)
template <bool F16>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float kv_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t kv_pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t kv_pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float kv_bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float kv_bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Four int8 codes -> two half pairs, exactly: the code with its sign bit flipped (0 .. 255) is the low byte of a half
// in [1024, 1280), from which 1152 is subtracted.
__device__ __forceinline__ void i8x4_to_f16(uint32_t x, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = x ^ 0x80808080u;
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 off = __half2half2(__ushort_as_half((unsigned short)0x6480));   // 1152
  const __half2 ra = __hsub2(*reinterpret_cast<const __half2*>(&a), off), rb = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
  lo = *reinterpret_cast<const uint32_t*>(&ra);
  hi = *reinterpret_cast<const uint32_t*>(&rb);
}
// Four int8 codes -> two bfloat16 pairs, exactly: the low seven bits sit in a bfloat16 in [128, 256), from which 128
// (or 256 where the sign bit is set) is subtracted.
__device__ __forceinline__ void i8x4_to_bf16(uint32_t x, uint32_t& lo, uint32_t& hi) {
  const uint32_t m = x & 0x7f7f7f7fu, s = x & 0x80808080u;
  const uint32_t a = __byte_perm(m, 0x43434343u, 0x4140), b = __byte_perm(m, 0x43434343u, 0x4342);
  const uint32_t c = __byte_perm(s, 0x43434343u, 0x4140), d = __byte_perm(s, 0x43434343u, 0x4342);
  const __nv_bfloat162 ra = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&c));
  const __nv_bfloat162 rb = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&b), *reinterpret_cast<const __nv_bfloat162*>(&d));
  lo = *reinterpret_cast<const uint32_t*>(&ra);
  hi = *reinterpret_cast<const uint32_t*>(&rb);
}

}  // namespace mq
