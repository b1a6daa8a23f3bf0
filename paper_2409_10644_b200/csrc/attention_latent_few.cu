// Tree attention over a latent cache for up to 16 query rows a sequence (single tokens of 16 heads, two of eight): bf16, rank
// 512, rotated part 64, on the warps' own matrix instructions.
//
//   S = Q K^T,  P = exp2(scale S - max),  O = O exp2(old max - max) + P V
//
// So few rows fill an eighth of what the kernel on tensor memory takes at a time; what counts for them is how soon the first keys
// are there and how short the way from the last ones to the result is.  A block takes all 16 rows and a range of keys, 64 at a
// time, two tiles in shared memory: one is used, one on its way.  Queries stay in registers.  Scores: a warp has eight keys over
// the whole row, in four independent sums; products with the values: 64 of the 512 channels.  The maximum of a tile and its
// weights pass through shared memory: three meetings of the block a tile (the tile is there, its maxima are, its weights are).  The
// ranges of a sequence are a cluster, which joins them through shared memory, or, where a sequence is long enough for more than 16, go
// through memory to a second kernel.  Weights are rounded to bf16, the type of the values that they multiply (half a step, 2^-8 of
// each); their sum is taken before that, in fp32.
//
// What bounds it: the chain of a tile (scores, maximum, weights, products: 1.6 us with two warps a scheduler, two and a half times
// what its loads take), so that it is taken where a block has few tiles, or where memory is the bound.  Rows come by bulk copies,
// one a row: fetched by all threads in 16-byte pieces their issue alone took 0.9 us a tile.  One token of 16 heads over 1001
// keys: 9.3 us in 16 blocks, 10.5 in eight, 17.8 on tensor memory.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "attention_tc_common.cuh"
#include "latent_pieces.cuh"

namespace cg = cooperative_groups;

namespace mcsd {

constexpr int kFewRows = 16, kFewKeys = 64, kFewThreads = 256, kFewRank = 512, kFewWidth = 576;
constexpr int kFewLd = kFewWidth + 8;      // elements of a row in shared memory: eight rows meet all banks
constexpr int kFewPLd = kFewKeys + 8;
constexpr int kFewVecs = kFewWidth / 8;    // 16-byte vectors of a row
constexpr int kFewCluster = 16;            // blocks of a cluster, at most
constexpr int kFewMost = 160;              // blocks of a sequence that are joined through memory, at most
constexpr int kFewSmem = (kFewRows * kFewLd + 2 * kFewKeys * kFewLd + kFewRows * kFewPLd) * 2 + (2 * 8 * kFewRows + 2 * kFewRows) * 4 + 32;
static_assert(kFewRows * kFewRank * 4 <= kFewKeys * kFewLd * 2, "results lie where keys were");
static_assert(kFewSmem <= 227 * 1024, "a block's shared memory");

__device__ __forceinline__ void ldm4(uint32_t* r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t* r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void few_copy(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// grid: (1, splits, B), the splits of a sequence a cluster where JOIN
template <bool JOIN>
__global__ void __launch_bounds__(kFewThreads, 1) latent_few_kernel(const __grid_constant__ LatentPieces g, float scale_log2, WorkspaceHeader* header) {
    extern __shared__ float4 raw4[];
    const LatentArgs& a = g.a;
    __nv_bfloat16* qs = reinterpret_cast<__nv_bfloat16*>(raw4);          // [16][kFewLd]
    __nv_bfloat16* ks = qs + kFewRows * kFewLd;                          // [2][64][kFewLd]
    __nv_bfloat16* ps = ks + 2 * kFewKeys * kFewLd;                      // [16][kFewPLd] weights of a tile
    float* red = reinterpret_cast<float*>(ps + kFewRows * kFewPLd);      // [2][warp][row]
    float* ml = red + 2 * 8 * kFewRows;                                  // [16] references, [16] sums
    unsigned long long* full = reinterpret_cast<unsigned long long*>(ml + 2 * kFewRows);
    int* abort_flag = reinterpret_cast<int*>(full + 2);                  // [2]
    const uint32_t q_a = smem_u32(qs), k_a = smem_u32(ks), p_a = smem_u32(ps);
    const int b = blockIdx.z, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    const int L = min(max(a.seq_lens[b], 0), a.L_max);
    const int nr = a.H * Nb;
    if (nr == 0) return;                                                 // (all blocks of a cluster alike)
    const int total = L + Nb, per = ((total + kFewKeys - 1) / kFewKeys + g.splits - 1) / g.splits * kFewKeys;
    const int k0 = min((long long)blockIdx.y * per, (long long)total), k1 = (int)min((long long)total, (long long)k0 + per);
    const __nv_bfloat16 *cache = static_cast<const __nv_bfloat16*>(a.cache) + (long long)b * a.L_max * kFewWidth,
                        *tree = static_cast<const __nv_bfloat16*>(a.tree) + (long long)b * a.N * kFewWidth;
    if (tid == 0) {
        mbar_init(&full[0], 1);
        mbar_init(&full[1], 1);
        abort_flag[0] = abort_flag[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    auto load_tile = [&](int buffer, int kb) {           // a row a copy, eight of them a warp
        if (tid == 0) mbar_expect_tx(&full[buffer], kFewKeys * kFewWidth * 2);
        if (lane < 8) {
            const int r = 8 * warp + lane, key = min(kb + r, k1 - 1);
            const __nv_bfloat16* src = key < L ? cache + (long long)key * kFewWidth : tree + (long long)(key - L) * kFewWidth;
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(k_a + (buffer * kFewKeys + r) * kFewLd * 2), "l"(src), "r"(kFewWidth * 2), "r"(smem_u32(&full[buffer])) : "memory");
        }
        __syncwarp();                                    // matrix instructions follow, which a warp executes together
    };
    if (k0 < k1) load_tile(0, k0);
    for (int i = tid; i < kFewRows * kFewVecs; i += kFewThreads) {
        const int r = i / kFewVecs, v = i - r * kFewVecs, rr = min(r, nr - 1), h = rr / Nb, n = rr - h * Nb;
        few_copy(q_a + (r * kFewLd + v * 8) * 2, static_cast<const __nv_bfloat16*>(a.q) + (((long long)b * a.H + h) * a.N + n) * kFewWidth + v * 8);
    }
    // this thread's rows of a product: row and row + 8, columns 2 (lane % 4) and the next
    const int row = lane >> 2, col = 2 * (lane & 3);
    const uint64_t *see0 = a.anc + (size_t)(min(row, nr - 1) % Nb) * a.words, *see1 = a.anc + (size_t)(min(row + 8, nr - 1) % Nb) * a.words;
    float o[8][4], m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
    uint32_t q[kFewWidth / 16][4];
    int t = 0;
    for (int kb = k0; kb < k1; kb += kFewKeys, ++t) {
        if (t == 0) asm volatile("cp.async.wait_all;" ::: "memory");                // the queries
        mbar_wait(&full[t & 1], (t >> 1) & 1, abort_flag, header, 30);
        __syncthreads();                                                            // and the other buffer has been read
        if (*(volatile int*)abort_flag) {              // (alike in all threads: whoever could set it next comes behind two meetings)
            // A wait ran out: no more copies, and this tile's, the only ones on their way, have as long again to come in before the
            // block leaves its memory.
            if (tid == 0) mbar_wait_slow(&full[t & 1], (t >> 1) & 1, abort_flag + 1, header, 31);
            break;
        }
        if (kb + kFewKeys < k1) load_tile((t + 1) & 1, kb + kFewKeys);
        if (t == 0) {
#pragma unroll
            for (int k = 0; k < kFewWidth / 16; ++k) ldm4(q[k], q_a + ((lane & 15) * kFewLd + 16 * k + 8 * (lane >> 4)) * 2);
        }
        const uint32_t tile = k_a + (t & 1) * kFewKeys * kFewLd * 2;
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
#pragma unroll
        for (int k = 0; k < kFewWidth / 32; ++k) {
            uint32_t f[4];
            ldm4(f, tile + ((8 * warp + (lane & 7)) * kFewLd + 32 * k + 8 * (lane >> 3)) * 2);
            mma16(s[2 * k & 3], q[2 * k], f[0], f[1]);
            mma16(s[(2 * k + 1) & 3], q[2 * k + 1], f[2], f[3]);
        }
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int key = kb + 8 * warp + col + (j & 1), node = key - L;
            bool see = key < k1;
            if (see && node >= 0) see = ((j < 2 ? see0 : see1)[node >> 6] >> (node & 63)) & 1;
            x[j] = see ? ((s[0][j] + s[1][j]) + (s[2][j] + s[3][j])) * scale_log2 : -INFINITY;
        }
        float t0 = fmaxf(x[0], x[1]), t1 = fmaxf(x[2], x[3]);
#pragma unroll
        for (int i = 1; i < 4; i <<= 1) {
            t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, i));
            t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, i));
        }
        float* const r = red + (t & 1) * 8 * kFewRows;
        if ((lane & 3) == 0) {
            r[warp * kFewRows + row] = t0;
            r[warp * kFewRows + row + 8] = t1;
        }
        __syncthreads();
        t0 = m0;
        t1 = m1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t0 = fmaxf(t0, r[i * kFewRows + row]);
            t1 = fmaxf(t1, r[i * kFewRows + row + 8]);
        }
        const float ref0 = t0 == -INFINITY ? 0.0f : t0, ref1 = t1 == -INFINITY ? 0.0f : t1;
        const float f0 = ex2_approx(m0 - ref0), f1 = ex2_approx(m1 - ref1);
        m0 = t0;
        m1 = t1;
        const float e0 = ex2_approx(x[0] - ref0), e1 = ex2_approx(x[1] - ref0), e2 = ex2_approx(x[2] - ref1), e3 = ex2_approx(x[3] - ref1);
        l0 = l0 * f0 + (e0 + e1);
        l1 = l1 * f1 + (e2 + e3);
        *reinterpret_cast<__nv_bfloat162*>(ps + row * kFewPLd + 8 * warp + col) = __floats2bfloat162_rn(e0, e1);
        *reinterpret_cast<__nv_bfloat162*>(ps + (row + 8) * kFewPLd + 8 * warp + col) = __floats2bfloat162_rn(e2, e3);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            o[i][0] *= f0;
            o[i][1] *= f0;
            o[i][2] *= f1;
            o[i][3] *= f1;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kFewKeys / 16; ++k) {
            uint32_t p[4];
            ldm4(p, p_a + ((lane & 15) * kFewPLd + 16 * k + 8 * (lane >> 4)) * 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t f[4];
                ldm4t(f, tile + ((16 * k + (lane & 15)) * kFewLd + 64 * warp + 16 * i + 8 * (lane >> 4)) * 2);
                mma16(o[2 * i], p, f[0], f[1]);
                mma16(o[2 * i + 1], p, f[2], f[3]);
            }
        }
    }
    // ---- this range's rows, unnormalised, references and sums
    asm volatile("cp.async.wait_all;" ::: "memory");                    // queries of a range without keys
#pragma unroll
    for (int i = 1; i < 4; i <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, i);
        l1 += __shfl_xor_sync(0xffffffffu, l1, i);
    }
    __syncthreads();                                                    // all products are done
    if ((lane & 3) == 0) {
        red[warp * kFewRows + row] = l0;
        red[warp * kFewRows + row + 8] = l1;
        if (warp == 0) {
            ml[row] = m0 * 0.6931471805599453f;
            ml[row + 8] = m1 * 0.6931471805599453f;
        }
    }
    float* os = reinterpret_cast<float*>(ks);                           // [16][512]
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        *reinterpret_cast<float2*>(os + row * kFewRank + 64 * warp + 8 * i + col) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(os + (row + 8) * kFewRank + 64 * warp + 8 * i + col) = make_float2(o[i][2], o[i][3]);
    }
    __syncthreads();
    if (tid < kFewRows) {
        float l = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) l += red[i * kFewRows + tid];
        ml[kFewRows + tid] = l;
    }
    if constexpr (JOIN) {
        cg::this_cluster().sync();
        latent_join_cluster<__nv_bfloat16, kFewCluster>(g, os, ml, kFewRows, b, Nb, 0, nr, tid, kFewThreads);
        cg::this_cluster().sync();                                      // others may still read this block's rows
    } else {
        __syncthreads();
        for (int i = tid; i < nr * (kFewRank / 2); i += kFewThreads) {
            const int r = i / (kFewRank / 2), d = 2 * (i % (kFewRank / 2)), h = r / Nb, n = r - h * Nb;
            float* p = g.part + ((long long)blockIdx.y * a.B * a.H * a.N + ((long long)b * a.H + h) * a.N + n) * (kFewRank + 2);
            *reinterpret_cast<float2*>(p + d) = *reinterpret_cast<const float2*>(os + r * kFewRank + d);
            if (d == 0) { p[kFewRank] = ml[r]; p[kFewRank + 1] = ml[kFewRows + r]; }
        }
    }
}

// Clusters of 1 .. kFewCluster blocks that run at a time.
struct FewFit {
    int clusters[kFewCluster + 1];
};
static cudaLaunchConfig_t few_config(int splits, int B, cudaStream_t stream, cudaLaunchAttribute* attr) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = (unsigned)splits; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1, splits, B);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = kFewSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = splits <= kFewCluster ? 1 : 0;
    return cfg;
}
static int few_fit(FewFit* out) {
    static std::mutex mu;
    static FewFit known[64];
    static bool have[64] = {};
    int dev = 0;
    MCSD_CUDA_CHECK(cudaGetDevice(&dev));
    std::lock_guard<std::mutex> lock(mu);
    if (dev >= 0 && dev < 64 && have[dev]) {
        *out = known[dev];
        return MCSD_OK;
    }
    // both attributes are per device; clusters of more than eight blocks are an option that a device may not have
    MCSD_CUDA_CHECK(cudaFuncSetAttribute(latent_few_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem));
    MCSD_CUDA_CHECK(cudaFuncSetAttribute(latent_few_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem));
    const bool large = cudaFuncSetAttribute(latent_few_kernel<true>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
    bool refused = !large;
    for (int s = 1; s <= kFewCluster; ++s) {
        cudaLaunchAttribute attr[1];
        const cudaLaunchConfig_t cfg = few_config(s, 1, nullptr, attr);
        int n = 0;
        if (s <= 8 || large) {
            const bool fits = cudaOccupancyMaxActiveClusters(&n, latent_few_kernel<true>, &cfg) == cudaSuccess;
            refused = refused || !fits;
            if (!fits) n = 0;
        }
        out->clusters[s] = n;
    }
    if (refused) (void)cudaGetLastError();                              // what was refused here is not an error of this call
    if (dev >= 0 && dev < 64) {
        known[dev] = *out;
        have[dev] = true;
    }
    return MCSD_OK;
}

// Blocks a sequence, or 0 where the kernel on tensor memory is sooner done.  In microseconds, from calls of 1 to 256 sequences of
// 100 to 131072 keys: here 2.5 and, for every wave of clusters, 5 and 1.63 a tile of 64 keys, and some for a join by few; there 18
// (less for one or two tiles, up to 5 more for pieces of long items) and 0.004 for each unit of its cut (10 a tile of 256 keys, 21
// a sequence), or the rows at 4.6 TB/s.  Here and there, 16 heads: one token over 100 keys 8.7 and 11, 1001: 9.3 and 17.8, 4000: 14.1
// and 20.0, 8000: 20.8 and 24.5, 32000: 59 in a cluster, 24.7 through memory, and 31, 131072: 44.6 and 53.5; 8 over 8000: 22.4 through
// memory and 31, 16 over 4000: 26 and 31, 64 over 2000: 38 and 44, 256 over 4000: 232 and 256.
int latent_few_splits(int B, int H, int N, int rank, int rot, int L_max, int dtype, int* splits) {
    *splits = 0;
    if (dtype != MCSD_BF16 || rank != kFewRank || rot != kFewWidth - kFewRank || (long long)H * N > kFewRows) return MCSD_OK;
    FewFit fit;
    const int st = few_fit(&fit);
    if (st != MCSD_OK) return st;
    const double tiles = std::ceil(((double)L_max + N) / kFewKeys);
    const double keys = L_max, there = std::min(18.0 + 0.0006 * std::min(keys, 8000.0), 9.5 + B * (1.0 + std::ceil(keys / 256.0)));
    double best = std::max(there + 0.004 * B * (21.0 + 10.0 * keys / 256.0), B * keys * kFewWidth * 2 / 4.6e6);
    for (int s = 1; s <= kFewCluster; ++s) {
        if (fit.clusters[s] < 1) continue;
        const double t = 2.5 + std::ceil((double)B / fit.clusters[s]) * (5.0 + 1.63 * std::ceil(tiles / s)) + 4.5 / s;
        if (t < best) {
            best = t;
            *splits = s;
        }
    }
    // more blocks a sequence, joined through memory by a second kernel: one wave, its scratch within the other kernel's
    const int many = std::min(fit.clusters[1] / B, kFewMost);
    if (many > kFewCluster && tiles >= many && latent_tc_shape(B, H, N, rank, rot, L_max, dtype) &&
        (size_t)many * B * H * N * (kFewRank + 2) * sizeof(float) <= latent_tc_workspace_bytes()) {
        const double t = 2.5 + 5.0 + 1.63 * std::ceil(tiles / many) + 8.0;
        if (t < best) *splits = many;
    }
    return MCSD_OK;
}
int tree_attention_latent_few(const LatentArgs& a, int splits, WorkspaceHeader* header, void* scratch, cudaStream_t stream) {
    LatentPieces g{};
    g.a = a;
    g.splits = splits;
    g.part = static_cast<float*>(scratch);
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = few_config(splits, a.B, stream, attr);
    const float scale_log2 = a.scale * 1.4426950408889634f;
    if (splits <= kFewCluster) {
        MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, latent_few_kernel<true>, g, scale_log2, header));
        count_launches(1);
        return MCSD_OK;
    }
    MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, latent_few_kernel<false>, g, scale_log2, header));
    count_launches(2);
    return latent_join_pieces(g, stream);
}

}  // namespace mcsd
