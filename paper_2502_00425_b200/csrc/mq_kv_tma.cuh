// Tensor maps and TMA loads of the cache's tensor-memory kernels (mq_kv_chunk.cu, mq_kv_weights_chunk.cu).
#pragma once

#include <cuda.h>

#include "mq_kv.cuh"
#include "mq_sm100.cuh"

namespace mq {

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

inline bool encode_bf16(CUtensorMap* map, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return encode_fn() && encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, es,
                                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The pages as a map [page][head][slot][channel], read in boxes of 64 channels x (a page's slots, at most `tile`)
// (a cache without pages: a map of one page, over any memory, that no coordinate in use reaches)
inline bool encode_pages(CUtensorMap* map, const void* base, const void* any, const KvView& c, int dim, int tile) {
  const int page = 1 << c.page_shift;
  if (c.n_pages == 0) base = any;
  const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)page, (cuuint64_t)c.n_kv_heads, (cuuint64_t)(c.n_pages > 0 ? c.n_pages : 1)};
  const cuuint64_t strides[3] = {(cuuint64_t)c.slot_stride, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride};
  const cuuint32_t box[4] = {64, (cuuint32_t)(page < tile ? page : tile), 1, 1};
  return encode_bf16(map, 4, base, dims, strides, box);
}
// The queries as a map [token][head][channel], read in boxes of 64 channels x the heads of a group x whole tokens: `rows` rows
inline bool encode_queries(CUtensorMap* map, const void* Q, int64_t ldq_bytes, int n_q_heads, int total_q, int group, int rows, int dim) {
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)n_q_heads, (cuuint64_t)total_q};
  const cuuint64_t strides[2] = {(cuuint64_t)dim * 2, (cuuint64_t)ldq_bytes};
  const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)(rows / group)};
  return encode_bf16(map, 3, Q, dims, strides, box);
}

}  // namespace mq
