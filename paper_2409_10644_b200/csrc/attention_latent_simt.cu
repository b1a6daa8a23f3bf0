// Tree attention over a latent cache on the CUDA cores, in fp32 throughout: fp32 tensors, and bf16 shapes that the
// tensor-core kernel does not take.
//
//   s[r][j] = scale <q_r, k_j>,   o_r = sum_j softmax_j(s[r][j]) k_j[:rank],   k_j one row of rank + rot values
//
// All heads of a sequence share the keys, so its H * n_active query rows are one matrix.  A block takes 32 of them and a
// range of keys, 32 at a time: the tile of rows lies in shared memory once, as keys and as values.  Scores: a thread has
// 2 x 2 of them; products: a warp has every row and 32-wide slices of the rank, so that a value read from shared memory
// meets 32 rows.  The running maximum and sum of the softmax are kept per row.  The keys are cut into pieces so that about
// two blocks run on a multiprocessor's turn; a second kernel joins the pieces.
#include <algorithm>
#include <cmath>

#include "latent.cuh"

namespace mcsd {

constexpr int kLsRows = 32, kLsKeys = 32, kLsThreads = 256;
constexpr int kLsBlocks = 296;             // blocks that a launch is cut into, about
constexpr int kLsSlices = kLatentMaxRank / 32 / 8;

struct LatentSimt {
    LatentArgs a;
    int row_blocks, splits, keys_per_split;
    float* part;                           // [splits][B][H * N][rank + 2], or unused with one split
};

template <typename T> __device__ __forceinline__ float ls_load(const T* p);
template <> __device__ __forceinline__ float ls_load(const float* p) { return __ldg(p); }
template <> __device__ __forceinline__ float ls_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
template <typename T> __device__ __forceinline__ void ls_store(T* p, float v);
template <> __device__ __forceinline__ void ls_store(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void ls_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// grid: (row blocks, splits, B)
template <typename T>
__global__ void __launch_bounds__(kLsThreads) latent_simt_kernel(const __grid_constant__ LatentSimt g) {
    extern __shared__ float4 raw4[];
    const LatentArgs& a = g.a;
    const int W = a.rank + a.rot, ld = W + 4;
    float* qs = reinterpret_cast<float*>(raw4);          // [32][ld]
    float* ks = qs + kLsRows * ld;                       // [32][ld]
    float* ps = ks + kLsKeys * ld;                       // [key][row], 36 floats a key
    float* stat = ps + kLsKeys * 36;                     // [32] factor of this tile
    const int b = blockIdx.z, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    const int L = min(max(a.seq_lens[b], 0), a.L_max);
    const int rows = a.H * Nb, r0 = blockIdx.x * kLsRows;
    const int total = L + Nb, k0 = blockIdx.y * g.keys_per_split, k1 = min(total, k0 + g.keys_per_split);
    if (r0 >= rows) return;
    const int nr = min(kLsRows, rows - r0);
    for (int r = warp; r < kLsRows; r += kLsThreads / 32) {
        const int rr = r0 + min(r, nr - 1), h = rr / Nb, n = rr - h * Nb;
        const T* src = static_cast<const T*>(a.q) + (((long long)b * a.H + h) * a.N + n) * W;
        for (int d = lane; d < W; d += 32) qs[r * ld + d] = ls_load(src + d);
    }
    float acc[kLsSlices][kLsRows];
#pragma unroll
    for (int s = 0; s < kLsSlices; ++s)
#pragma unroll
        for (int r = 0; r < kLsRows; ++r) acc[s][r] = 0.0f;
    float m[4], l[4];                                    // rows 4 warp .. 4 warp + 3
#pragma unroll
    for (int i = 0; i < 4; ++i) { m[i] = -INFINITY; l[i] = 0.0f; }
    const int ty = tid >> 4, tx = tid & 15;              // scores: rows ty, ty + 16, keys tx, tx + 16
    for (int kb = k0; kb < k1; kb += kLsKeys) {
        __syncthreads();
        for (int j = warp; j < kLsKeys; j += kLsThreads / 32) {
            const int key = min(kb + j, k1 - 1);
            const T* src = key < L ? static_cast<const T*>(a.cache) + ((long long)b * a.L_max + key) * W
                                   : static_cast<const T*>(a.tree) + ((long long)b * a.N + (key - L)) * W;
            for (int d = lane; d < W; d += 32) ks[j * ld + d] = ls_load(src + d);
        }
        __syncthreads();
        float s00 = 0, s01 = 0, s10 = 0, s11 = 0;
        {
            const float4 *q0 = reinterpret_cast<const float4*>(qs + ty * ld), *q1 = reinterpret_cast<const float4*>(qs + (ty + 16) * ld);
            const float4 *c0 = reinterpret_cast<const float4*>(ks + tx * ld), *c1 = reinterpret_cast<const float4*>(ks + (tx + 16) * ld);
#pragma unroll 4
            for (int d = 0; d < W / 4; ++d) {
                const float4 x = q0[d], y = q1[d], u = c0[d], v = c1[d];
                s00 += x.x * u.x; s00 += x.y * u.y; s00 += x.z * u.z; s00 += x.w * u.w;
                s01 += x.x * v.x; s01 += x.y * v.y; s01 += x.z * v.z; s01 += x.w * v.w;
                s10 += y.x * u.x; s10 += y.y * u.y; s10 += y.z * u.z; s10 += y.w * u.w;
                s11 += y.x * v.x; s11 += y.y * v.y; s11 += y.z * v.z; s11 += y.w * v.w;
            }
        }
        ps[tx * 36 + ty] = s00;
        ps[(tx + 16) * 36 + ty] = s01;
        ps[tx * 36 + ty + 16] = s10;
        ps[(tx + 16) * 36 + ty + 16] = s11;
        __syncthreads();
        const int key = kb + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                    // a lane a key
            const int r = 4 * warp + i, rr = r0 + min(r, nr - 1), n = rr % Nb;
            bool see = key < k1;
            if (see && key >= L) see = (a.anc[(size_t)n * a.words + ((key - L) >> 6)] >> ((key - L) & 63)) & 1;
            const float s = see ? ps[lane * 36 + r] * a.scale : -INFINITY;
            float mx = s;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.0f : mn;
            const float f = m[i] == -INFINITY ? 0.0f : expf(m[i] - ref);
            const float p = see ? expf(s - ref) : 0.0f;
            float sum = p;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l[i] = l[i] * f + sum;
            m[i] = mn;
            ps[lane * 36 + r] = p;
            if (lane == 0) stat[r] = f;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kLsSlices; ++s) {
            const int d = (warp + 8 * s) * 32 + lane;
            if ((warp + 8 * s) * 32 < a.rank) {
#pragma unroll
                for (int r = 0; r < kLsRows; ++r) acc[s][r] *= stat[r];
                for (int j = 0; j < kLsKeys; ++j) {
                    const float v = ks[j * ld + d];
#pragma unroll
                    for (int r = 0; r < kLsRows; r += 4) {
                        const float4 p = *reinterpret_cast<const float4*>(ps + j * 36 + r);
                        acc[s][r] += p.x * v; acc[s][r + 1] += p.y * v; acc[s][r + 2] += p.z * v; acc[s][r + 3] += p.w * v;
                    }
                }
            }
        }
    }
    // one piece: the result; several: unnormalised values, maximum and sum
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (lane == 0) { ps[4 * warp + i] = m[i]; stat[4 * warp + i] = l[i]; }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kLsSlices; ++s) {
        const int d = (warp + 8 * s) * 32 + lane;
        if (d >= a.rank) continue;
#pragma unroll
        for (int r = 0; r < kLsRows; ++r) {
            if (r >= nr) continue;
            const int rr = r0 + r, h = rr / Nb, n = rr - h * Nb;
            const long long row = ((long long)b * a.H + h) * a.N + n;
            if (g.splits == 1) {
                ls_store(static_cast<T*>(a.out) + row * a.rank + d, stat[r] > 0.0f ? acc[s][r] / stat[r] : acc[s][r]);
            } else {
                float* p = g.part + ((long long)blockIdx.y * a.B * a.H * a.N + row) * (a.rank + 2);
                p[d] = acc[s][r];
                if (d == 0) { p[a.rank] = ps[r]; p[a.rank + 1] = stat[r]; }
            }
        }
    }
}

// grid: (H * N, B); joins the pieces of a row in their order
template <typename T>
__global__ void __launch_bounds__(128) latent_simt_join_kernel(const __grid_constant__ LatentSimt g) {
    const LatentArgs& a = g.a;
    const int b = blockIdx.y, n = blockIdx.x % a.N;
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    if (n >= Nb) return;
    const long long row = (long long)b * a.H * a.N + blockIdx.x, stride = (long long)a.B * a.H * a.N * (a.rank + 2);
    const float* p = g.part + row * (a.rank + 2);
    float m = -INFINITY;
    for (int s = 0; s < g.splits; ++s) m = fmaxf(m, p[s * stride + a.rank]);
    float l = 0.0f;
    for (int s = 0; s < g.splits; ++s) {
        const float ms = p[s * stride + a.rank];
        if (ms != -INFINITY) l += p[s * stride + a.rank + 1] * expf(ms - m);
    }
    for (int d = threadIdx.x; d < a.rank; d += 128) {
        float o = 0.0f;
        for (int s = 0; s < g.splits; ++s) {
            const float ms = p[s * stride + a.rank];
            if (ms != -INFINITY) o += p[s * stride + d] * expf(ms - m);
        }
        ls_store(static_cast<T*>(a.out) + row * a.rank + d, l > 0.0f ? o / l : o);
    }
}

static int split_of(int B, int H, int N, int L_max, int* row_blocks, int* keys_per_split) {
    *row_blocks = (int)(((long long)H * N + kLsRows - 1) / kLsRows);
    const long long blocks = (long long)*row_blocks * B, total = (long long)L_max + N, tiles = (total + kLsKeys - 1) / kLsKeys;
    const long long want = std::max(1LL, std::min(tiles, (kLsBlocks + blocks - 1) / blocks));
    const long long per = (tiles + want - 1) / want;
    *keys_per_split = (int)std::min(per * kLsKeys, 0x7fffffffLL - kLsKeys);
    return (int)((tiles + per - 1) / per);
}

size_t latent_simt_workspace_bytes(int B, int H, int N, int rank, int L_max) {
    int rb, ks;
    const int splits = split_of(B, H, N, L_max, &rb, &ks);
    return splits > 1 ? (size_t)splits * B * H * N * (rank + 2) * sizeof(float) : 0;
}

template <typename T>
static int run_simt(const LatentSimt& g, cudaStream_t stream) {
    const int smem = ((kLsRows + kLsKeys) * (g.a.rank + g.a.rot + 4) + kLsKeys * 36 + 32) * (int)sizeof(float);
    MCSD_CUDA_CHECK(cudaFuncSetAttribute(latent_simt_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    latent_simt_kernel<T><<<dim3(g.row_blocks, g.splits, g.a.B), kLsThreads, smem, stream>>>(g);
    MCSD_CUDA_CHECK(cudaGetLastError());
    if (g.splits > 1) {
        latent_simt_join_kernel<T><<<dim3(g.a.H * g.a.N, g.a.B), 128, 0, stream>>>(g);
        MCSD_CUDA_CHECK(cudaGetLastError());
    }
    count_launches(g.splits > 1 ? 2 : 1);
    return MCSD_OK;
}

int tree_attention_latent_simt(const LatentArgs& a, void* scratch, cudaStream_t stream) {
    LatentSimt g{};
    g.a = a;
    g.splits = split_of(a.B, a.H, a.N, a.L_max, &g.row_blocks, &g.keys_per_split);
    g.part = static_cast<float*>(scratch);
    return a.dtype == MCSD_F32 ? run_simt<float>(g, stream) : run_simt<__nv_bfloat16>(g, stream);
}

}  // namespace mcsd
