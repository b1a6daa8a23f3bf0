// Arguments of the norm-and-rotation kernel (norm_rope.cu).
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace mcsd {

struct NormRopeArgs {
    const void *q_in, *k_in, *v_in;
    long long q_batch, q_token, k_batch, k_token, v_batch, v_token;   // strides in elements
    const void *q_weight, *k_weight;                                  // [D] or NULL
    float eps;
    const double* freqs;                                              // [rot_dim / 2], radians per position
    int rot_dim;
    bool interleaved;
    const int32_t *seq_lens, *depth, *n_active;
    void *q_out, *k_out, *v_out;
    int B, H_q, H_kv, N;
};

}  // namespace mcsd
