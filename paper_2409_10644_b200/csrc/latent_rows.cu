// Rows of a latent cache from a target layer's projections, and the commit of accepted rows.
//
//   row = (c, r):  c = x[:rank] * rsqrt(mean(x[:rank]^2) + eps) * w,   r = x[rank:] rotated by the token's position
//   q[..., rank:] = the heads' rotated parts, likewise;   angle_i = position * freq[i]
//
// Every element is read once and written once, so memory bounds the rows of a prompt (512 + 64 values and 32 heads of 64: 8191
// tokens move 86 MB in 16 us, 5.3 TB/s) and the launch those of a token (3.0 us).  A block takes a few tokens: it reduces their
// angles once, as a fraction of a turn in 64 bits (a far position leaves no bits for the angle in 32), and all heads of a token
// use them; a thread turns eight pairs at a time from 16-byte vectors.  Statistics and rotations are in 32 bits, one rounding
// at the store.
//
// A commit is bound by its launch and two loads that wait for one another (where a node's row lies, then the row): 3.7 us
// for 2 layers of 4 sequences, 8.5 us for 32 of 32, whose rows alone would take 1.7.
#include <algorithm>

#include "latent.cuh"

namespace mcsd {

constexpr int kRowThreads = 256;
constexpr int kRowTokens = 4;          // tokens of a block at most

struct LatentRowArgs {
    const void *latent, *q_in, *weight;
    long long latent_batch, latent_token, q_batch, q_token, q_head;   // strides in elements
    const double* freqs;
    const int32_t *seq_lens, *depth, *n_active, *row_start;
    void *rows, *q;
    int B, H, N, rank, rot, L_rows, interleaved, tokens;
    float eps;
    bool vec_latent, vec_q, vec_rows, vec_qout, vec_w;               // 16-byte accesses allowed
};

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(float x) { return x; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }

// eight consecutive elements
template <typename T>
struct alignas(16) Eight {
    T t[8];
    __device__ __forceinline__ void load(const T* p, bool vec) {
        if (vec) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(t)[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = p[i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return to_f<T>(t[i]); }
};
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v, bool vec) {
    alignas(16) T t[8];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<__nv_bfloat162*>(t)[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = from_f<T>(v[i]);
    }
    if (vec) {
        constexpr int n = sizeof(T) * 8 / 16;
#pragma unroll
        for (int i = 0; i < n; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = t[i];
    }
}

// Pairs 8 v .. 8 v + 7 of a rotated part: read, then turned and stored.  cs holds (cos, sin) of every pair.
template <typename T>
struct Turn8 {
    Eight<T> a, b;
    __device__ __forceinline__ void load(const T* src, int rot, int v, bool interleaved, bool vec) {
        a.load(src + (interleaved ? 16 * v : 8 * v), vec);
        b.load(src + (interleaved ? 16 * v + 8 : rot / 2 + 8 * v), vec);
    }
    __device__ __forceinline__ void store(T* dst, const float2* cs, int rot, int v, bool interleaved, bool vec) const {
        float x[8], y[8];
        float2 w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 c = reinterpret_cast<const float4*>(cs + 8 * v)[i];
            w[2 * i] = make_float2(c.x, c.y);
            w[2 * i + 1] = make_float2(c.z, c.w);
        }
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 c = w[i], d = w[4 + i];
                x[2 * i] = a[2 * i] * c.x - a[2 * i + 1] * c.y;
                x[2 * i + 1] = a[2 * i + 1] * c.x + a[2 * i] * c.y;
                y[2 * i] = b[2 * i] * d.x - b[2 * i + 1] * d.y;
                y[2 * i + 1] = b[2 * i + 1] * d.x + b[2 * i] * d.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 c = w[i];
                x[i] = a[i] * c.x - b[i] * c.y;
                y[i] = b[i] * c.x + a[i] * c.y;
            }
        }
        store8(dst + (interleaved ? 16 * v : 8 * v), x, vec);
        store8(dst + (interleaved ? 16 * v + 8 : rot / 2 + 8 * v), y, vec);
    }
};

// grid: (ceil(N / tokens), B).  VEC: all accesses are 16-byte ones
template <typename T, bool VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kRowThreads) latent_rows_kernel(const __grid_constant__ LatentRowArgs a) {
    __shared__ __align__(16) float2 cs[kRowTokens][kLatentMaxRot / 2];      // (a row: 16-byte aligned)
    const int b = blockIdx.y, n0 = blockIdx.x * a.tokens;
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    const int nt = min(a.tokens, Nb - n0);
    if (nt <= 0) return;
    const int half = a.rot / 2, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int W = a.rank + a.rot;
    // the heads' parts are on their way while the angles are reduced and the latent part is normalised: a thread takes the
    // same vector of every G-th head, counted through the block's tokens (without a division: the kernel is bound by its
    // instructions before it is by memory)
    constexpr int kAhead = 4 / sizeof(T);
    const int per_head = half / 8, G = per_head > 0 ? kRowThreads / per_head : 1;
    const int g = per_head > 0 ? threadIdx.x / per_head : 0, v8 = threadIdx.x - g * per_head;
    const bool heads = a.q && g < G;
    const T* const q_src = static_cast<const T*>(a.q_in) + b * a.q_batch + n0 * a.q_token;
    T* const q_dst = static_cast<T*>(a.q) + ((long long)b * a.H * a.N + n0) * W + a.rank;
    const long long head_step = (long long)a.N * W;
    auto next = [&](int& t, int& h) {
        h += G;
        while (h >= a.H && t < nt) { h -= a.H; ++t; }
    };
    int ft = 0, fh = g - G, pt = 0, ph = g - G;        // token and head that are fetched, and put
    next(ft, fh);
    next(pt, ph);
    auto fetch = [&](Turn8<T>& x) {
        if (ft < nt) x.load(q_src + ft * a.q_token + fh * a.q_head, a.rot, v8, INTERLEAVED, VEC || a.vec_q);
        next(ft, fh);
    };
    auto put = [&](const Turn8<T>& x) {
        if (pt < nt) x.store(q_dst + ph * head_step + pt * W, cs[pt], a.rot, v8, INTERLEAVED, VEC || a.vec_qout);
        next(pt, ph);
    };
    Turn8<T> ahead[kAhead];
    if (heads) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) fetch(ahead[j]);
    }
    for (int i = threadIdx.x ^ (kRowThreads / 2); i < nt * half; i += kRowThreads) {   // by the warps without a latent part first
        const int t = i / half, j = i - t * half, n = n0 + t;
        const double pos = (double)a.seq_lens[b] + (double)(a.depth ? a.depth[n] : n);
        double turns = pos * a.freqs[j] * 0.15915494309189535;      // 1 / 2 pi
        turns -= rint(turns);
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        cs[t][j] = make_float2(c, s);
    }
    // one warp a token: the latent part needs no angles
    const T* x = nullptr;
    T* dst = nullptr;
    if (a.rows && warp < nt) {
        const int n = n0 + warp;
        const long long row = (long long)n + (a.row_start ? a.row_start[b] : 0);
        x = static_cast<const T*>(a.latent) + b * a.latent_batch + n * a.latent_token;
        if (row >= 0 && row < a.L_rows) dst = static_cast<T*>(a.rows) + ((long long)b * a.L_rows + row) * W;
        if (dst) {
            Eight<T> v[kLatentMaxRank / 256];
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kLatentMaxRank / 256; ++k) {
                const int e = (k * 32 + lane) * 8;
                if (e < a.rank) {
                    v[k].load(x + e, VEC || a.vec_latent);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += v[k][i] * v[k][i];
                }
            }
            float r = 1.0f;
            if (a.weight) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                r = rsqrtf(sum / (float)a.rank + a.eps);
            }
#pragma unroll
            for (int k = 0; k < kLatentMaxRank / 256; ++k) {
                const int e = (k * 32 + lane) * 8;
                if (e < a.rank) {
                    float y[8];
                    Eight<T> w;
                    if (a.weight) w.load(static_cast<const T*>(a.weight) + e, VEC || a.vec_w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = a.weight ? v[k][i] * r * w[i] : v[k][i];
                    store8(dst + e, y, VEC || a.vec_rows);
                }
            }
        }
    }
    __syncthreads();
    if (dst && lane < half / 8) {
        Turn8<T> r;
        r.load(x + a.rank, a.rot, lane, INTERLEAVED, VEC || a.vec_latent);
        r.store(dst + a.rank, cs[warp], a.rot, lane, INTERLEAVED, VEC || a.vec_rows);
    }
    if (heads) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) put(ahead[j]);
        while (pt < nt) {
            Turn8<T> x;
            fetch(x);
            put(x);
        }
    }
}

// ------------------------------------------------------------------ commit
// Rows of the winning root and the accepted nodes behind the prefix of every layer (Fig. 1 step 6).  One launch: a cluster
// of blocks takes a sequence and shares its layers; its first block grows the length once all of them have read it.
constexpr int kCommitCluster = 8, kLatentCommitThreads = 256;

__global__ void __cluster_dims__(kCommitCluster, 1, 1) __launch_bounds__(kLatentCommitThreads)
commit_latent_kernel(void* const* __restrict__ cache_layers, const void* const* __restrict__ tree_layers, int n_layers,
                     int32_t* __restrict__ seq_lens, const int32_t* __restrict__ accept_len, const int32_t* __restrict__ out_nodes,
                     const int32_t* __restrict__ best_root, int n_levels, int N, int L_max, int row_bytes) {
    const int b = blockIdx.y, rank = blockIdx.x;
    const int L = min(max(seq_lens[b], 0), L_max);
    const int acc = min(max(accept_len[b], 0), n_levels);
    const int count = min(1 + acc, L_max - L);
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // the length has been read
    const int vecs = row_bytes / 16, per_layer = count * vecs;
    const int layers = (n_layers - rank + kCommitCluster - 1) / kCommitCluster;
    constexpr int kFlight = 4;                          // vectors of a thread on their way at a time
    for (int i = threadIdx.x; i < layers * per_layer; i += kFlight * kLatentCommitThreads) {
        const char* src[kFlight];
        char* dst[kFlight];
        uint4 x[kFlight];
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            src[j] = nullptr;
            const int at = i + j * kLatentCommitThreads;
            if (at >= layers * per_layer) continue;
            const int k = at / per_layer, rest = at - k * per_layer, layer = rank + k * kCommitCluster;
            const int t = rest / vecs, v = rest - t * vecs;
            const int node = t == 0 ? best_root[b] : out_nodes[(size_t)b * n_levels + (t - 1)];
            if (node < 0 || node >= N) continue;                    // malformed verify output: leave the row alone
            src[j] = static_cast<const char*>(tree_layers[layer]) + ((size_t)b * N + node) * row_bytes + v * 16;
            dst[j] = static_cast<char*>(cache_layers[layer]) + ((size_t)b * L_max + L + t) * row_bytes + v * 16;
        }
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (src[j] && (reinterpret_cast<uintptr_t>(src[j]) & 15u) == 0) x[j] = *reinterpret_cast<const uint4*>(src[j]);
            else if (src[j])
                for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t*>(&x[j])[e] = reinterpret_cast<const uint16_t*>(src[j])[e];
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (src[j] && (reinterpret_cast<uintptr_t>(dst[j]) & 15u) == 0) *reinterpret_cast<uint4*>(dst[j]) = x[j];
            else if (src[j])
                for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t*>(dst[j])[e] = reinterpret_cast<const uint16_t*>(&x[j])[e];
    }
    __syncwarp();                                       // lanes leave the loop after different trips; the wait is the warp's
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0 && threadIdx.x == 0) seq_lens[b] = min(L_max, L + 1 + acc);
}

template <typename T>
static void launch_latent_rows(const LatentRowArgs& a, dim3 grid, cudaStream_t s) {
    const bool vec = (a.vec_latent && a.vec_rows && (a.vec_w || !a.weight) || !a.rows) && (a.vec_q && a.vec_qout || !a.q);
    if (vec && a.interleaved) latent_rows_kernel<T, true, true><<<grid, kRowThreads, 0, s>>>(a);
    else if (vec) latent_rows_kernel<T, true, false><<<grid, kRowThreads, 0, s>>>(a);
    else if (a.interleaved) latent_rows_kernel<T, false, true><<<grid, kRowThreads, 0, s>>>(a);
    else latent_rows_kernel<T, false, false><<<grid, kRowThreads, 0, s>>>(a);
}
static bool vec_ok(const void* p, std::initializer_list<long long> strides, int elt) {
    if (reinterpret_cast<uintptr_t>(p) & 15u) return false;
    for (long long s : strides)
        if ((s * elt) % 16) return false;
    return true;
}

}  // namespace mcsd

extern "C" int mcsd_latent_rows(const void* latent_in, const void* q_in, const int64_t* strides, const void* weight, float eps,
                                const double* freqs, int interleaved, const int32_t* seq_lens, const int32_t* depth,
                                const int32_t* n_active, const int32_t* row_start, void* rows, int L_rows, void* q, int B, int H,
                                int N, int rank, int rot, int dtype, void* stream) {
    if (!strides || !seq_lens || (!rows && !q)) return MCSD_ERR_NULL;
    if ((rows && !latent_in) || (q && rot > 0 && !q_in) || (rot > 0 && !freqs)) return MCSD_ERR_NULL;
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (B < 1 || B > 65535 || N < 1 || (long long)B * N > 0x7fffffffLL || !mcsd::latent_widths_ok(rank, rot)) return MCSD_ERR_BAD_SHAPE;
    if (rows && L_rows < 1) return MCSD_ERR_BAD_SHAPE;
    if (q && (H < 1 || H > 65535)) return MCSD_ERR_BAD_SHAPE;
    if (!(eps >= 0.0f)) return MCSD_ERR_BAD_SHAPE;
    const int elt = dtype == MCSD_F32 ? 4 : 2;
    mcsd::LatentRowArgs a{};
    a.latent = latent_in; a.q_in = q_in; a.weight = weight;
    a.latent_batch = strides[0]; a.latent_token = strides[1];
    a.q_batch = strides[2]; a.q_token = strides[3]; a.q_head = strides[4];
    a.freqs = freqs;
    a.seq_lens = seq_lens; a.depth = depth; a.n_active = n_active; a.row_start = row_start;
    a.rows = rows; a.q = rot > 0 ? q : nullptr;
    a.B = B; a.H = H; a.N = N; a.rank = rank; a.rot = rot; a.L_rows = L_rows; a.interleaved = interleaved != 0;
    a.eps = eps;
    if (!a.rows && !a.q) return MCSD_OK;                           // queries without a rotated part: nothing to do
    a.vec_latent = mcsd::vec_ok(latent_in, {a.latent_batch, a.latent_token}, elt);
    a.vec_q = mcsd::vec_ok(q_in, {a.q_batch, a.q_token, a.q_head}, elt);
    a.vec_rows = mcsd::vec_ok(rows, {}, elt);
    a.vec_qout = mcsd::vec_ok(q, {}, elt);
    a.vec_w = mcsd::vec_ok(weight, {}, elt);
    // more tokens a block share its start, fewer fill the multiprocessors: one or four cost 3.4 or 5.9 us at 64 tokens of 128
    // heads, 3.4 or 3.5 at 256 of 32, 3.8 or 3.6 at 512, 32.7 or 16.0 at 8192 (there two 21.5, eight 17.2)
    a.tokens = (long long)B * N >= 512 ? mcsd::kRowTokens : 1;
    const dim3 grid((N + a.tokens - 1) / a.tokens, B);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == MCSD_F32) mcsd::launch_latent_rows<float>(a, grid, s);
    else mcsd::launch_latent_rows<__nv_bfloat16>(a, grid, s);
    MCSD_CUDA_CHECK(cudaGetLastError());
    mcsd::count_launches(1);
    return MCSD_OK;
}

extern "C" int mcsd_commit_latent(void* const* cache_layers, const void* const* tree_layers, int n_layers, int32_t* seq_lens,
                                  const int32_t* accept_len, const int32_t* out_nodes, const int32_t* best_root, int n_levels, int B,
                                  int N, int width, int L_max, int dtype, void* stream) {
    if (!cache_layers || !tree_layers || !seq_lens || !accept_len || !out_nodes || !best_root) return MCSD_ERR_NULL;
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (n_layers < 1 || n_layers > 65535 || B < 1 || B > 65535 || N < 1 || N > MCSD_MAX_NODES || L_max < 1 || n_levels < 1 || n_levels > N)
        return MCSD_ERR_BAD_SHAPE;
    if (width < 32 || width > mcsd::kLatentMaxRank + mcsd::kLatentMaxRot || width % 16) return MCSD_ERR_BAD_SHAPE;
    const int row_bytes = width * (dtype == MCSD_F32 ? 4 : 2);
    mcsd::commit_latent_kernel<<<dim3(mcsd::kCommitCluster, B), mcsd::kLatentCommitThreads, 0, static_cast<cudaStream_t>(stream)>>>(
        cache_layers, tree_layers, n_layers, seq_lens, accept_len, out_nodes, best_root, n_levels, N, L_max, row_bytes);
    MCSD_CUDA_CHECK(cudaGetLastError());
    mcsd::count_launches(1);
    return MCSD_OK;
}
