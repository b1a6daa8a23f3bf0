// Internal interface between the C ABI entry point of tree attention and its kernels.
#pragma once

#include "common.cuh"

namespace mcsd {

// What an attention workspace holds: the status line, the counters with which the blocks of a tensor-core launch tell one
// another that a piece of a cut work item is done (zero between launches), then scratch, which may hold anything between
// launches.  The place of the counters depends on nothing, so that calls of any type, shape, cache and kernel may follow one
// another on one workspace: a work item is cut between consecutive blocks and a block starts at most one cut item, so the
// items are known by the block that starts them (kCountersPerBlock each: one per softmax group of the kernel over dense caches).
constexpr int kTcMaxBlocks = 160;                    // thread blocks of a launch, at most (one per multiprocessor)
constexpr int kCountersPerBlock = 4;
struct AttentionWorkspace {
    WorkspaceHeader header;
    int counters[kTcMaxBlocks * kCountersPerBlock];
};
static_assert(sizeof(AttentionWorkspace) % 256 == 0, "scratch starts on a 256-byte line");

struct AttentionArgs {
    const void* q;
    const void* k_cache;
    const void* v_cache;
    const void* k_tree;
    const void* v_tree;
    void* out;
    const int32_t* seq_lens;
    const int32_t* n_active;
    const uint64_t* anc;
    int words;
    int B, H, N, D, L_max;   // H: query heads
    float scale;
    int dtype;
    int G;                   // query heads per key/value head (1: multi-head attention); key/value tensors have H / G heads
    const void* kv4 = nullptr;   // the prefix cache as 4-bit pages (kv4.cuh) instead of k_cache and v_cache
};

// CUDA-core path (fp32, or bf16 shapes the tensor-core kernel does not take)
size_t simt_workspace_bytes(int B, int H, int N, int D, int L_max);
int tree_attention_simt(const AttentionArgs& a, void* scratch, cudaStream_t stream);

// tcgen05 tensor-core path: bf16, D = 128
bool tc_shape_supported(int B, int H, int G, int N, int D, int L_max, int dtype);   // shape and dtype alone
bool tc_supported(const AttentionArgs& a);
size_t tc_workspace_bytes(int B, int H, int N, int D, int L_max);
int tc_bounded_wait_selftest(WorkspaceHeader* header, long long limit_cycles, int where, cudaStream_t stream);
int tc_plan_host(int B, int H, int G, int N, int L_max, const int32_t* seq_lens, const int32_t* n_active, int grid,
                 long long* first_tile, long long* info, int n_probe, const long long* probe_tiles, long long* probe_out);
int tree_attention_tc(const AttentionArgs& a, AttentionWorkspace* workspace, void* scratch, size_t scratch_bytes,
                      cudaStream_t stream);

// tcgen05 path over a 4-bit cache: bf16, D = 128, the shapes of the tensor-core kernel above
bool kv4_tc_shape(int B, int H, int G, int N, int D, int L_max, int dtype);
size_t kv4_tc_workspace_bytes();
int tree_attention_kv4_tc(const AttentionArgs& a, AttentionWorkspace* workspace, void* scratch, cudaStream_t stream);

}  // namespace mcsd
