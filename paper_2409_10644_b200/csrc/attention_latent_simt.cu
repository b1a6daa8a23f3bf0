// Tree attention over a latent cache on the CUDA cores, in fp32 throughout: fp32 tensors, and bf16 shapes that the
// tensor-core kernel does not take.
//
//   s[r][j] = scale <q_r, k_j>,   o_r = sum_j softmax_j(s[r][j]) k_j[:rank],   k_j one row of rank + rot values
//
// All heads of a sequence share the keys, so its H * n_active query rows are one matrix.  A block takes 32 of them and a
// range of keys, 32 at a time: the tile of rows lies in shared memory once, as keys and as values.  Scores: a thread has 8 x 4
// of them over an eighth of the row, so that 12 vectors read from shared memory meet in 128 products.  Products with the
// values: a warp has 64 columns and 32 rows, or fewer rows where the rank has fewer columns than eight warps take.  The
// running maximum and sum of the softmax are kept per row.  The keys are cut into pieces so that about two blocks run on a
// multiprocessor's turn; up to eight pieces are a cluster, which joins them through shared memory, more are joined by a second
// kernel (two sequences of 131 + 15 keys, 60 rows of 128 + 32: 20.5 us with that, 9.4 in a
// cluster).  Shared memory and the products bound it: 25 TFLOP/s at 512 + 64, 256 x 45 rows over 4000 keys, of 74 nominal.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "latent_pieces.cuh"

namespace cg = cooperative_groups;

namespace mcsd {

constexpr int kLsRows = 32, kLsKeys = 32, kLsThreads = 256;
constexpr int kLsBlocks = 296;             // blocks that a launch is cut into, about
constexpr int kLsScores = 36;              // floats of a key's weights
constexpr int ls_smem(int width) { return ((kLsRows + kLsKeys) * width + kLsKeys * kLsScores + kLsRows) * (int)sizeof(float); }
constexpr int kLsSmemMost = ls_smem(kLatentMaxRank + kLatentMaxRot);
static_assert(kLsSmemMost <= 227 * 1024, "a block's shared memory");

template <typename T> __device__ __forceinline__ float ls_load(const T* p);
template <> __device__ __forceinline__ float ls_load(const float* p) { return __ldg(p); }
template <> __device__ __forceinline__ float ls_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
// One row of W values to shared memory, by a warp; four vectors of a lane are on their way at a time.
template <typename T>
__device__ __forceinline__ void ls_row(float* dst, const T* src, int W, int lane, bool vec) {
    if (!vec) {
        for (int d = lane; d < W; d += 32) dst[d] = ls_load(src + d);
    } else if constexpr (sizeof(T) == 4) {
        for (int d = 4 * lane; d < W; d += 128)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + d)), "l"(src + d) : "memory");
    } else {
#pragma unroll 2
        for (int d = 8 * lane; d < W; d += 256) {
            const uint4 x = __ldg(reinterpret_cast<const uint4*>(src + d));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
            float v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
            *reinterpret_cast<float4*>(dst + d) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(dst + d + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
}

// grid: (row blocks, splits, B), splits a cluster where JOIN.  ROWS: rows of a warp's products, 32 columns of 64 for 8 warps
template <typename T, int ROWS, bool JOIN>
__global__ void __launch_bounds__(kLsThreads) latent_simt_kernel(const __grid_constant__ LatentPieces g) {
    extern __shared__ float4 raw4[];
    const LatentArgs& a = g.a;
    const int W = a.rank + a.rot;
    float* qs = reinterpret_cast<float*>(raw4);          // [32][W]
    float* ks = qs + kLsRows * W;                        // [32][W]
    float* ps = ks + kLsKeys * W;                        // [key][row], 36 floats a key
    float* stat = ps + kLsKeys * kLsScores;              // [32] factor of this tile
    const int b = blockIdx.z, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    const int L = min(max(a.seq_lens[b], 0), a.L_max);
    const int rows = a.H * Nb, r0 = blockIdx.x * kLsRows;
    const int total = L + Nb, k0 = blockIdx.y * g.keys_per_split, k1 = min(total, k0 + g.keys_per_split);
    if (r0 >= rows) return;                              // (all blocks of a cluster alike)
    const int nr = min(kLsRows, rows - r0);
    for (int r = warp; r < kLsRows; r += kLsThreads / 32) {
        const int rr = r0 + min(r, nr - 1), h = rr / Nb, n = rr - h * Nb;
        ls_row(qs + r * W, static_cast<const T*>(a.q) + (((long long)b * a.H + h) * a.N + n) * W, W, lane, g.vec);
    }
    constexpr int kWarps = 8 * ROWS / 32;                // warps side by side along the columns
    const int row0 = warp / kWarps * ROWS, col = warp % kWarps * 64 + 2 * lane;
    float2 acc[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) acc[r] = make_float2(0.0f, 0.0f);
    float m[4], l[4];                                    // rows 4 warp .. 4 warp + 3
#pragma unroll
    for (int i = 0; i < 4; ++i) { m[i] = -INFINITY; l[i] = 0.0f; }
    // scores: rows 8 ty .., keys tx, tx + 8, .., every eighth vector of the row from dq on
    const int dq = lane & 7, ty = warp >> 1, tx = (warp & 1) * 4 + (lane >> 3);
    for (int kb = k0; kb < k1; kb += kLsKeys) {
        __syncthreads();
        for (int j = warp; j < kLsKeys; j += kLsThreads / 32) {
            const int key = min(kb + j, k1 - 1);
            const T* src = key < L ? static_cast<const T*>(a.cache) + ((long long)b * a.L_max + key) * W
                                   : static_cast<const T*>(a.tree) + ((long long)b * a.N + (key - L)) * W;
            ls_row(ks + j * W, src, W, lane, g.vec);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        float s[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
        for (int d = 4 * dq; d < W; d += 32) {
            float4 k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(ks + (tx + 8 * j) * W + d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 q = *reinterpret_cast<const float4*>(qs + (8 * ty + i) * W + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] += q.x * k[j].x;
                    s[i][j] += q.y * k[j].y;
                    s[i][j] += q.z * k[j].z;
                    s[i][j] += q.w * k[j].w;
                }
            }
        }
        // summed over the eight lanes, each of which is left with one row
#pragma unroll
        for (int o = 4; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < o; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float send = dq & o ? s[i][j] : s[i + o][j], keep = dq & o ? s[i + o][j] : s[i][j];
                    s[i][j] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
#pragma unroll
        for (int j = 0; j < 4; ++j) ps[(tx + 8 * j) * kLsScores + 8 * ty + dq] = s[0][j];
        __syncthreads();
        const int key = kb + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                    // a lane a key
            const int r = 4 * warp + i, rr = r0 + min(r, nr - 1), n = rr % Nb;
            bool see = key < k1;
            if (see && key >= L) see = (a.anc[(size_t)n * a.words + ((key - L) >> 6)] >> ((key - L) & 63)) & 1;
            const float x = see ? ps[lane * kLsScores + r] * a.scale : -INFINITY;
            float mx = x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.0f : mn;
            const float f = m[i] == -INFINITY ? 0.0f : expf(m[i] - ref);
            const float p = see ? expf(x - ref) : 0.0f;
            float sum = p;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l[i] = l[i] * f + sum;
            m[i] = mn;
            ps[lane * kLsScores + r] = p;
            if (lane == 0) stat[r] = f;
        }
        __syncthreads();
        if (col < a.rank) {
            if (kb > k0) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float f = stat[row0 + r];
                    acc[r].x *= f;
                    acc[r].y *= f;
                }
            }
#pragma unroll 4
            for (int j = 0; j < kLsKeys; ++j) {
                const float2 v = *reinterpret_cast<const float2*>(ks + j * W + col);
#pragma unroll
                for (int r = 0; r < ROWS; r += 4) {
                    const float4 p = *reinterpret_cast<const float4*>(ps + j * kLsScores + row0 + r);
                    acc[r].x += p.x * v.x; acc[r].y += p.x * v.y;
                    acc[r + 1].x += p.y * v.x; acc[r + 1].y += p.y * v.y;
                    acc[r + 2].x += p.z * v.x; acc[r + 2].y += p.z * v.y;
                    acc[r + 3].x += p.w * v.x; acc[r + 3].y += p.w * v.y;
                }
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");      // queries of a piece without keys
    __syncthreads();
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { ps[4 * warp + i] = m[i]; ps[kLsRows + 4 * warp + i] = l[i]; }
    }
    if constexpr (JOIN) {
        // unnormalised rows to shared memory, where every block of the cluster joins some of them
        float* os = qs;                                  // [32][rank]
        if (col < a.rank) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) *reinterpret_cast<float2*>(os + (row0 + r) * a.rank + col) = acc[r];
        }
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        latent_join_cluster<T, kLatentCluster>(g, os, ps, kLsRows, b, Nb, r0, nr, tid, kLsThreads);
        cluster.sync();                                  // others may still read this block's rows
    } else {
        __syncthreads();
        if (col < a.rank) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (row0 + r >= nr) continue;
                const int rr = r0 + row0 + r, h = rr / Nb, n = rr - h * Nb;
                const long long row = ((long long)b * a.H + h) * a.N + n;
                float* p = g.part + ((long long)blockIdx.y * a.B * a.H * a.N + row) * (a.rank + 2);
                *reinterpret_cast<float2*>(p + col) = acc[r];
                if (col == 0) { p[a.rank] = ps[row0 + r]; p[a.rank + 1] = ps[kLsRows + row0 + r]; }
            }
        }
    }
}

// grid: (H * N, B, 128 channels each); joins the pieces of a row in their order, every fourth by a quarter of the threads
constexpr int kJoinThreads = 512, kJoinParts = kJoinThreads / 128;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) latent_join_kernel(const __grid_constant__ LatentPieces g) {
    __shared__ float weight[kLsBlocks];
    __shared__ float red[kJoinThreads / 32];
    __shared__ float2 parts[kJoinParts][128];
    const LatentArgs& a = g.a;
    const int b = blockIdx.y, n = blockIdx.x % a.N, tid = threadIdx.x, part = tid >> 7;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    if (n >= Nb) return;
    const long long row = (long long)b * a.H * a.N + blockIdx.x, stride = (long long)a.B * a.H * a.N * (a.rank + 2);
    const float* p = g.part + row * (a.rank + 2);
    float m = -INFINITY;
    for (int s = tid; s < g.splits; s += kJoinThreads) {
        weight[s] = p[s * stride + a.rank];
        m = fmaxf(m, weight[s]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((tid & 31) == 0) red[tid >> 5] = m;
    __syncthreads();
    for (int i = 0; i < kJoinThreads / 32; ++i) m = fmaxf(m, red[i]);
    for (int s = tid; s < g.splits; s += kJoinThreads) weight[s] = weight[s] == -INFINITY ? 0.0f : expf(weight[s] - m);
    __syncthreads();
    const int d = blockIdx.z * 128 + (tid & 127);
    float l = 0.0f, o = 0.0f;
    if (d < a.rank) {
#pragma unroll 8
        for (int s = part; s < g.splits; s += kJoinParts) {
            const float x = p[s * stride + d], y = p[s * stride + a.rank + 1];
            l += y * weight[s];
            o += x * weight[s];
        }
    }
    parts[part][tid & 127] = make_float2(l, o);
    __syncthreads();
    if (part > 0 || d >= a.rank) return;
    for (int k = 1; k < kJoinParts; ++k) {
        l += parts[k][tid].x;
        o += parts[k][tid].y;
    }
    latent_store(static_cast<T*>(a.out) + row * a.rank + d, l > 0.0f ? o / l : o);
}
int latent_join_pieces(const LatentPieces& g, cudaStream_t stream) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(g.a.H * g.a.N, g.a.B, (g.a.rank + 127) / 128);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (g.a.dtype == MCSD_F32) MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, latent_join_kernel<float>, g));
    else MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, latent_join_kernel<__nv_bfloat16>, g));
    return MCSD_OK;
}

static int split_of(int B, int H, int N, int L_max, int* row_blocks, int* keys_per_split) {
    *row_blocks = (int)(((long long)H * N + kLsRows - 1) / kLsRows);
    const long long blocks = (long long)*row_blocks * B, total = (long long)L_max + N, tiles = (total + kLsKeys - 1) / kLsKeys;
    long long want = std::max(1LL, std::min(tiles, (kLsBlocks + blocks - 1) / blocks));
    if (want <= 2 * kLatentCluster) want = std::min(want, (long long)kLatentCluster);   // one launch
    const long long per = (tiles + want - 1) / want;
    *keys_per_split = (int)std::min(per * kLsKeys, 0x7fffffffLL - kLsKeys);
    return (int)((tiles + per - 1) / per);
}

int latent_simt_splits(int B, int H, int N, int L_max) {
    int rb, ks;
    return split_of(B, H, N, L_max, &rb, &ks);
}
size_t latent_simt_workspace_bytes(int B, int H, int N, int rank, int L_max) {
    const int splits = latent_simt_splits(B, H, N, L_max);
    return splits > kLatentCluster ? (size_t)splits * B * H * N * (rank + 2) * sizeof(float) : 0;
}

template <typename T, int ROWS, bool JOIN>
static int run_simt(const LatentPieces& g, cudaStream_t stream) {
    // one instance serves many widths, and what it may take is the process's: the most that any of them takes, so that no host thread
    // lowers it between another one's setting and launch
    MCSD_CUDA_CHECK(cudaFuncSetAttribute(latent_simt_kernel<T, ROWS, JOIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLsSmemMost));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = (unsigned)g.splits; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(g.row_blocks, g.splits, g.a.B);
    cfg.blockDim = dim3(kLsThreads);
    cfg.dynamicSmemBytes = ls_smem(g.a.rank + g.a.rot);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = JOIN ? 1 : 0;
    MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, latent_simt_kernel<T, ROWS, JOIN>, g));
    count_launches(JOIN ? 1 : 2);
    return JOIN ? MCSD_OK : latent_join_pieces(g, stream);
}
template <typename T>
static int pick_simt(const LatentPieces& g, cudaStream_t stream) {
    const bool join = g.splits <= kLatentCluster;
    if (g.a.rank > 256) return join ? run_simt<T, 32, true>(g, stream) : run_simt<T, 32, false>(g, stream);
    if (g.a.rank > 128) return join ? run_simt<T, 16, true>(g, stream) : run_simt<T, 16, false>(g, stream);
    if (g.a.rank > 64) return join ? run_simt<T, 8, true>(g, stream) : run_simt<T, 8, false>(g, stream);
    return join ? run_simt<T, 4, true>(g, stream) : run_simt<T, 4, false>(g, stream);
}

int tree_attention_latent_simt(const LatentArgs& a, void* scratch, cudaStream_t stream) {
    LatentPieces g{};
    g.a = a;
    g.splits = split_of(a.B, a.H, a.N, a.L_max, &g.row_blocks, &g.keys_per_split);
    g.part = static_cast<float*>(scratch);
    g.vec = ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.cache) | reinterpret_cast<uintptr_t>(a.tree)) & 15u) == 0;
    return a.dtype == MCSD_F32 ? pick_simt<float>(g, stream) : pick_simt<__nv_bfloat16>(g, stream);
}

}  // namespace mcsd
