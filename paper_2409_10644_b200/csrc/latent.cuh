// Internal interface of the operators over a latent cache (one shared row of `rank` + `rot` values a token): the row and
// commit kernels (latent_rows.cu), the entry point of tree attention (attention_latent.cu) and its two kernels.
#pragma once

#include <cuda_bf16.h>

#include "attention.cuh"

namespace mcsd {

constexpr int kLatentMaxRank = 512, kLatentMaxRot = 128;

// ranks and rotated parts that every latent operator takes (rows are then whole 16-byte vectors in both types)
inline bool latent_widths_ok(int rank, int rot) {
    return rank >= 32 && rank <= kLatentMaxRank && rank % 32 == 0 && rot >= 0 && rot <= kLatentMaxRot && rot % 16 == 0;
}

struct LatentArgs {
    const void *q, *cache, *tree;
    void* out;
    const int32_t *seq_lens, *n_active;
    const uint64_t* anc;
    int words;
    int B, H, N, rank, rot, L_max;
    float scale;
    int dtype;
};

// CUDA-core kernel: fp32, and bf16 shapes or alignments that the tensor-core kernel does not take
int latent_simt_splits(int B, int H, int N, int L_max);
size_t latent_simt_workspace_bytes(int B, int H, int N, int rank, int L_max);
int tree_attention_latent_simt(const LatentArgs& a, void* scratch, cudaStream_t stream);

// warp-level matrix instructions: up to 16 query rows a sequence, bf16, rank 512, rotated part 64, tensors on 16-byte boundaries
// (blocks a sequence, 0 where it is not taken)
int latent_few_splits(int B, int H, int N, int rank, int rot, int L_max, int dtype, int* splits);
int tree_attention_latent_few(const LatentArgs& a, int splits, WorkspaceHeader* header, void* scratch, cudaStream_t stream);

// tcgen05 kernel: bf16, rank 512, rotated part 64, tensors on 16-byte boundaries
bool latent_tc_shape(int B, int H, int N, int rank, int rot, int L_max, int dtype);
size_t latent_tc_workspace_bytes();
bool latent_tc_set_patience(long long cycles);       // negative: the default, which is the most
int tree_attention_latent_tc(const LatentArgs& a, AttentionWorkspace* workspace, void* scratch, cudaStream_t stream);

}  // namespace mcsd
