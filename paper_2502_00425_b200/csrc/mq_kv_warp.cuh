// What the kernels for few query rows share (mq_kv_attn.cu, mq_kv_weights.cu): a warp streams tiles of 16 keys from the pages
// into a ring of its own by TMA, and multiplies them, as the rows of an mma.sync tile, with up to 8 kN query rows.
#pragma once

#include "mq_kv_sched.cuh"
#include "mq_kv_tma.cuh"

namespace mq {

constexpr int kStreamWarps = 4;                      // warps of a CTA
constexpr int kStreamThreads = kStreamWarps * 32;
constexpr int kStreamTile = 16 * kStreamWarps;       // keys of a tile of the work line: 16 per warp

// K (or V) rows of 16 keys in shared memory, as TMA leaves them: blocks of 128 bytes per row with the 16-byte pieces of a row
// exchanged by the row's number (64-byte rows: by the pair's), so that the rows one load instruction touches lie in different banks.
template <int kD, bool kI8>
struct KeyTile {
  static constexpr int kRow = kD * (kI8 ? 1 : 2);    // bytes of a cached row
  static constexpr int kBlocks = kRow > 128 ? kRow / 128 : 1;
  static constexpr int kBytes = 16 * kRow;
  // offset of 16-byte piece c of row r
  static __device__ __forceinline__ uint32_t piece(int r, int c) {
    if (kRow == 64) {
      const uint32_t off = (uint32_t)r * 64u + (uint32_t)c * 16u;
      return off ^ (((off >> 7) & 3u) << 4);
    }
    return (uint32_t)(c >> 3) * 2048u + (uint32_t)r * 128u + (((uint32_t)c ^ (uint32_t)r) & 7u) * 16u;
  }
  static __device__ __forceinline__ void load(uint32_t dst, const CUtensorMap* map, int slot, int head, int page, uint64_t* bar) {
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) tma_load_4d(dst + (uint32_t)b * 2048u, map, b * (kI8 ? 128 : 64), slot, head, page, bar);
  }
};

// The pages as a map of boxes of 16 keys, laid out as KeyTile says.  A cache without pages has a map of one page that no
// coordinate in use reaches.
inline bool encode_key_tiles(CUtensorMap* map, const void* base, const void* any, const KvView& c, int dim, bool i8) {
  const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)1 << c.page_shift, (cuuint64_t)c.n_kv_heads, (cuuint64_t)(c.n_pages > 0 ? c.n_pages : 1)};
  const cuuint64_t strides[3] = {(cuuint64_t)c.slot_stride, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)(i8 ? dim : 64), 16, 1, 1}, es[4] = {1, 1, 1, 1};
  return encode_fn() &&
         encode_fn()(map, i8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(c.n_pages > 0 ? base : any), dims,
                     strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, i8 && dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Query row as column `quad` of a B operand: qf[k] = channels of step k.  fac[e] = what turns the scores of rows 2 t4 + e into
// log2 units.  An int8 cache takes fp16 queries, brought into range by a power of two per row, in the channel order that lets a thread read contiguous codes: step k, position (2 t4, 2 t4 + 1, 2 t4 + 8,
// 2 t4 + 9) is channel t4 * D/4 + 4 k + 0 .. 3.  In two parts, so that the loads can travel while something else is done.
template <int kD, bool kI8>
__device__ __forceinline__ void fetch_query(const uint8_t* q, bool ok, int t4, uint32_t (&qf)[kD / 16][2]) {
#pragma unroll
  for (int k = 0; k < kD / 16; ++k) {
    if (kI8) {
      const uint2 w = ok ? *reinterpret_cast<const uint2*>(q + (t4 * (kD / 4) + 4 * k) * 2) : make_uint2(0u, 0u);
      qf[k][0] = w.x;
      qf[k][1] = w.y;
    } else {
      const int c = (k * 16 + 2 * t4) * 2;
      qf[k][0] = ok ? *reinterpret_cast<const uint32_t*>(q + c) : 0u;
      qf[k][1] = ok ? *reinterpret_cast<const uint32_t*>(q + c + 16) : 0u;
    }
  }
}
template <int kD, bool kI8>
__device__ __forceinline__ void finish_query(int t4, float base_fac, uint32_t (&qf)[kD / 16][2], float (&fac)[2]) {
  constexpr int kSteps = kD / 16;
  fac[0] = fac[1] = base_fac;
  if (kI8) {
    float m = 0.0f;
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) m = fmaxf(m, fmaxf(fabsf(kv_bf16_lo(qf[k][e])), fabsf(kv_bf16_hi(qf[k][e]))));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    // the power of two that brings the row's largest magnitude into [2^14, 2^15), the highest that fp16 has room for: the 8
    // bits of a channel are all kept down to 2^-31 of the largest, and what smaller ones lose is below 2^-39 of it.  (An
    // infinity stays one either way; the last bound keeps the factor itself finite.)
    const int e2 = m > 0.0f && m < INFINITY ? max((int)((__float_as_uint(m) >> 23) & 255) - 127 - 14, -126) : 0;
    const float f = exp2f((float)-e2), back = base_fac * exp2f((float)e2);
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) qf[k][e] = kv_pack_f16(kv_bf16_lo(qf[k][e]) * f, kv_bf16_hi(qf[k][e]) * f);
    fac[0] = __shfl_sync(0xffffffffu, back, 8 * t4);
    fac[1] = __shfl_sync(0xffffffffu, back, 8 * t4 + 4);
  }
}

// Pages of a warp's tiles i = 0, 1, .. (the tile's first key is first_key + i * kStreamTile): lane l holds that of tile
// base + l, so the table is read once per 32 tiles.
struct PageWindow {
  const int32_t* table;
  int first_key, shift, n, base, mine;
  __device__ __forceinline__ void fetch(int lane) {
    const int i = base + lane;
    mine = i < n ? table[(first_key + i * kStreamTile) >> shift] : 0;
  }
  __device__ __forceinline__ PageWindow(const int32_t* t, int first, int sh, int tiles, int lane) : table(t), first_key(first), shift(sh), n(tiles), base(0) {
    fetch(lane);
  }
  __device__ __forceinline__ int page(int i, int lane) {   // every lane asks for the same i, in order
    if (i - base >= 32) {
      base = i;
      fetch(lane);
    }
    return __shfl_sync(0xffffffffu, mine, i - base);
  }
};

// S^T = K Q^T of 16 keys: s[nt] = (key quad, row 2 t4), (quad, 2 t4 + 1), (quad + 8, 2 t4), (quad + 8, 2 t4 + 1) of block nt.
// Two chains of products each, so that they overlap.
template <int kD, bool kI8, int kN>
__device__ __forceinline__ void key_scores(uint32_t kt, int lane, const uint32_t (&qf)[kN][kD / 16][2], float (&s)[kN][4]) {
  using T = KeyTile<kD, kI8>;
  float s2[kN][4];
#pragma unroll
  for (int nt = 0; nt < kN; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[nt][e] = s2[nt][e] = 0.0f;
  if (!kI8) {
#pragma unroll
    for (int k = 0; k < kD / 16; ++k) {
      uint32_t a[4];
      ldsm_x4(kt + T::piece(lane & 15, 2 * k + (lane >> 4)), a);
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) mma_16816<false>((k & 1) ? s2[nt] : s[nt], a, qf[nt][k][0], qf[nt][k][1]);
    }
  } else {
    constexpr int kLoads = kD / 64;   // 16-byte loads per key row and thread
    const int quad = lane >> 2, t4 = lane & 3;
#pragma unroll
    for (int c = 0; c < kLoads; ++c) {
      uint32_t x[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(x[j][0]), "=r"(x[j][1]), "=r"(x[j][2]), "=r"(x[j][3]) : "r"(kt + T::piece(quad + 8 * j, t4 * kLoads + c)) : "memory");
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t a[4];
        i8x4_to_f16(x[0][w], a[0], a[2]);
        i8x4_to_f16(x[1][w], a[1], a[3]);
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) mma_16816<true>((w & 1) ? s2[nt] : s[nt], a, qf[nt][4 * c + w][0], qf[nt][4 * c + w][1]);
      }
    }
  }
#pragma unroll
  for (int nt = 0; nt < kN; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[nt][e] += s2[nt][e];
}

}  // namespace mq
