// C ABI entry point of tree attention over a latent cache: argument checks and the choice of kernel.
#include <algorithm>

#include "latent.cuh"

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static int check_latent(int B, int H, int N, int rank, int rot, int L_max, int dtype) {
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (B < 1 || H < 1 || N < 1 || N > MCSD_MAX_NODES || L_max < 0 || L_max > (1 << 30) || (long long)B * H > 65535) return MCSD_ERR_BAD_SHAPE;
    return mcsd::latent_widths_ok(rank, rot) ? MCSD_OK : MCSD_ERR_BAD_SHAPE;
}

// The kernel of a call, or a status; *splits: blocks a sequence of the one for few rows, pieces of the keys of the one on the CUDA cores.
static int choose(int B, int H, int N, int rank, int rot, int L_max, int dtype, bool aligned, int* splits) {
    *splits = 0;
    if (aligned) {
        const int st = mcsd::latent_few_splits(B, H, N, rank, rot, L_max, dtype, splits);
        if (st != MCSD_OK) return st;
        if (*splits > 0) return MCSD_PATH_FEW_ROWS;
        if (mcsd::latent_tc_shape(B, H, N, rank, rot, L_max, dtype)) return MCSD_PATH_TENSOR_CORE;
    }
    *splits = mcsd::latent_simt_splits(B, H, N, L_max);
    return MCSD_PATH_CUDA_CORE;
}

extern "C" int mcsd_tree_attention_latent_path(int B, int H, int N, int rank, int rot, int L_max, int dtype, int* splits) {
    const int st = check_latent(B, H, N, rank, rot, L_max, dtype);
    if (st != MCSD_OK) return st;
    int s = 0;
    const int path = choose(B, H, N, rank, rot, L_max, dtype, true, &s);
    if (splits) *splits = s;
    return path;
}

extern "C" size_t mcsd_tree_attention_latent_workspace_bytes(int B, int H, int N, int rank, int rot, int L_max, int dtype) {
    if (check_latent(B, H, N, rank, rot, L_max, dtype) != MCSD_OK) return 0;
    size_t scratch = mcsd::latent_simt_workspace_bytes(B, H, N, rank, L_max);      // bf16 tensors off a 16-byte boundary
    if (mcsd::latent_tc_shape(B, H, N, rank, rot, L_max, dtype)) scratch = std::max(scratch, mcsd::latent_tc_workspace_bytes());
    return sizeof(mcsd::AttentionWorkspace) + mcsd::align_up(scratch, 256);
}

extern "C" int mcsd_tree_attention_latent(const void* q, const void* cache, const void* tree, void* out, const int32_t* seq_lens,
                                          const int32_t* n_active, const uint64_t* anc, int words, int B, int H, int N, int rank,
                                          int rot, int L_max, float softmax_scale, int dtype, void* workspace,
                                          size_t workspace_bytes, void* stream) {
    if (!q || !tree || !out || !seq_lens || !anc || !workspace) return MCSD_ERR_NULL;
    const int st = check_latent(B, H, N, rank, rot, L_max, dtype);
    if (st != MCSD_OK) return st;
    if (L_max > 0 && !cache) return MCSD_ERR_NULL;
    if (words < (N + 63) / 64 || words > MCSD_MAX_WORDS) return MCSD_ERR_BAD_SHAPE;
    if (workspace_bytes < mcsd_tree_attention_latent_workspace_bytes(B, H, N, rank, rot, L_max, dtype)) return MCSD_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return MCSD_ERR_BAD_SHAPE;
    const mcsd::LatentArgs a{q, cache, tree, out, seq_lens, n_active, anc, words, B, H, N, rank, rot, L_max, softmax_scale, dtype};
    auto* ws = static_cast<mcsd::AttentionWorkspace*>(workspace);
    const bool aligned = aligned16(q) && aligned16(cache) && aligned16(tree) && aligned16(out);
    int splits = 0;
    const int path = choose(B, H, N, rank, rot, L_max, dtype, aligned, &splits);
    if (path < 0) return path;
    if (path == MCSD_PATH_FEW_ROWS) return mcsd::tree_attention_latent_few(a, splits, &ws->header, ws + 1, static_cast<cudaStream_t>(stream));
    if (path == MCSD_PATH_TENSOR_CORE) return mcsd::tree_attention_latent_tc(a, ws, ws + 1, static_cast<cudaStream_t>(stream));
    return mcsd::tree_attention_latent_simt(a, ws + 1, static_cast<cudaStream_t>(stream));
}

extern "C" int mcsd_selftest_latent_patience(long long cycles) {
    return mcsd::latent_tc_set_patience(cycles) ? MCSD_OK : MCSD_ERR_BAD_SHAPE;
}
