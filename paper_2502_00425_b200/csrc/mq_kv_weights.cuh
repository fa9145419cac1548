// Arguments of the two kernels that accumulate the keys' softmax weights (mq_kv_weights.cu, mq_kv_weights_chunk.cu).
#pragma once

#include "mq_kv.cuh"

namespace mq {

struct WeightParams {
  const uint8_t* Q;
  int64_t ldq;   // bytes
  KvBatchView b;
  KvView c;
  int max_q, n_q_heads;
  FastDiv group;   // query heads per key/value head
  float scale;
  const float* lse;
  const float* W_in;
  float* W_out;
  int64_t seq_stride, head_stride;
  int w_keys;        // entries of a row of W: a sequence with more keys is reported, and keys behind it are left out
  int32_t* status;   // device int32[2] or nullptr
};

// many query rows, on tensor memory; most_units: an upper bound of its units of 128 keys
int launch_kv_weights_chunk(const WeightParams& p, int dim, bool i8, int64_t most_units, cudaStream_t st);

}  // namespace mq
