// Tree attention over a latent cache by blocks that take a range of the keys: what they leave, and how it is joined.
#pragma once

#include <cooperative_groups.h>

#include <cmath>

#include "latent.cuh"

namespace mcsd {

constexpr int kLatentCluster = 8;          // pieces that a cluster joins; more go through memory

struct LatentPieces {
    LatentArgs a;
    int row_blocks, splits, keys_per_split;
    bool vec;                              // 16-byte loads
    float* part;                           // [splits][B][H * N][rank + 2], unused where a cluster joins
};
// Joins the pieces that lie in part, in their order (a launch of its own).
int latent_join_pieces(const LatentPieces& g, cudaStream_t stream);

template <typename T> __device__ __forceinline__ void latent_store(T* p, float v);
template <> __device__ __forceinline__ void latent_store(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void latent_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// Joins the rows r0 .. r0 + nr - 1 of sequence b in a cluster of g.splits (at most MOST) blocks along the keys, each every splits-th row, between
// two meetings of the cluster: os [rows][rank] unnormalised values of a block, ml its references (natural logarithms), then,
// `rows` further, its sums.
template <typename T, int MOST>
__device__ __forceinline__ void latent_join_cluster(const LatentPieces& g, float* os, float* ml, int rows, int b, int Nb, int r0, int nr, int tid, int threads) {
    const LatentArgs& a = g.a;
    const auto cluster = cooperative_groups::this_cluster();
    const int vecs = a.rank / 4, mine = (nr - (int)blockIdx.y + g.splits - 1) / g.splits;
    for (int i = tid; i < mine * vecs; i += threads) {
        const int r = (int)blockIdx.y + i / vecs * g.splits, d = 4 * (i % vecs);
        float pm[MOST], pl[MOST], top = -INFINITY, sum = 0.0f;
        float4 v[MOST], o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            if (k >= g.splits) continue;
            const float* peer = cluster.map_shared_rank(ml, k);
            pm[k] = peer[r];
            pl[k] = peer[rows + r];
            v[k] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(os, k) + r * a.rank + d);
        }
#pragma unroll
        for (int k = 0; k < MOST; ++k)
            if (k < g.splits) top = fmaxf(top, pm[k]);
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            if (k >= g.splits || pm[k] == -INFINITY) continue;
            const float f = expf(pm[k] - top);
            sum += pl[k] * f;
            o.x += v[k].x * f; o.y += v[k].y * f; o.z += v[k].z * f; o.w += v[k].w * f;
        }
        const int rr = r0 + r, h = rr / Nb, n = rr - h * Nb;
        T* out = static_cast<T*>(a.out) + (((long long)b * a.H + h) * a.N + n) * a.rank + d;
        const float y[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) latent_store(out + j, sum > 0.0f ? y[j] / sum : y[j]);
    }
}

}  // namespace mcsd
