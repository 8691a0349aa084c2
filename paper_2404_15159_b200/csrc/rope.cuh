// Arguments of the rotary kernels.
#pragma once

#include "common.cuh"

namespace mixlora {

struct RopeArgs {
  const void *q, *k;              // [tokens, heads, head_dim], `*_stride` elements from token to token
  void *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;
  const int32_t* positions;       // [tokens], or NULL: the token's index
  const double* inv_freq;         // [pairs] radians per position
  float amplitude;
  int tokens, q_heads, k_heads, head_dim;
  int pairs;                      // rotary_dim / 2
  int copied;                     // values behind rotary_dim that have to be copied (0 in place)
  int backward;
  int shares;                     // warps that share a token's heads
};

cudaError_t launch_rope_frequencies(int pairs, double theta, int scaling, double factor, double low, double high,
                                    double original, double* out, cudaStream_t st);
cudaError_t launch_rope(RopeArgs p, bool bf16_mode, bool interleaved, cudaStream_t st);

}  // namespace mixlora
