// Rows of a latent cache from a target layer's projections, and the commit of accepted rows.
//
//   row = (c, r):  c = x[:rank] * rsqrt(mean(x[:rank]^2) + eps) * w,   r = x[rank:] rotated by the token's position
//   q[..., rank:] = the heads' rotated parts, likewise;   angle_i = position * freq[i]
//
// Every element is read once and written once, so memory bounds the rows of a prompt and the launch those of a token.  A
// block takes a few tokens: it reduces their angles once, as a fraction of a turn in 64 bits (a far position leaves no bits
// for the angle in 32), and all heads of a token use them; a thread turns eight pairs at a time from 16-byte vectors.
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
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = from_f<T>(v[i]);
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
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 c = cs[8 * v + i], d = cs[8 * v + 4 + i];
                x[2 * i] = a[2 * i] * c.x - a[2 * i + 1] * c.y;
                x[2 * i + 1] = a[2 * i + 1] * c.x + a[2 * i] * c.y;
                y[2 * i] = b[2 * i] * d.x - b[2 * i + 1] * d.y;
                y[2 * i + 1] = b[2 * i + 1] * d.x + b[2 * i] * d.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 c = cs[8 * v + i];
                x[i] = a[i] * c.x - b[i] * c.y;
                y[i] = b[i] * c.x + a[i] * c.y;
            }
        }
        store8(dst + (interleaved ? 16 * v : 8 * v), x, vec);
        store8(dst + (interleaved ? 16 * v + 8 : rot / 2 + 8 * v), y, vec);
    }
};

// grid: (ceil(N / tokens), B)
template <typename T>
__global__ void __launch_bounds__(kRowThreads) latent_rows_kernel(const __grid_constant__ LatentRowArgs a) {
    __shared__ float2 cs[kRowTokens][kLatentMaxRot / 2];
    const int b = blockIdx.y, n0 = blockIdx.x * a.tokens;
    const int Nb = a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N;
    const int nt = min(a.tokens, Nb - n0);
    if (nt <= 0) return;
    const int half = a.rot / 2, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int W = a.rank + a.rot;
    // the heads' parts are on their way while the angles are reduced and the latent part is normalised
    constexpr int kAhead = 4 / sizeof(T);
    const int per_head = half / 8, per_token = a.H * per_head, parts = a.q ? nt * per_token : 0;
    auto part = [&](int i, int& t, int& h, int& v) {
        t = i / per_token;
        const int k = i - t * per_token;
        h = k / per_head;
        v = k - h * per_head;
    };
    auto fetch = [&](Turn8<T>& x, int i) {
        int t, h, v;
        part(i, t, h, v);
        x.load(static_cast<const T*>(a.q_in) + b * a.q_batch + (n0 + t) * a.q_token + h * a.q_head, a.rot, v, a.interleaved, a.vec_q);
    };
    auto put = [&](const Turn8<T>& x, int i) {
        int t, h, v;
        part(i, t, h, v);
        T* o = static_cast<T*>(a.q) + (((long long)b * a.H + h) * a.N + n0 + t) * W + a.rank;
        x.store(o, cs[t], a.rot, v, a.interleaved, a.vec_qout);
    };
    Turn8<T> ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if ((int)threadIdx.x + j * kRowThreads < parts) fetch(ahead[j], threadIdx.x + j * kRowThreads);
    for (int i = threadIdx.x; i < nt * half; i += kRowThreads) {
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
                    v[k].load(x + e, a.vec_latent);
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
                    if (a.weight) w.load(static_cast<const T*>(a.weight) + e, a.vec_w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = a.weight ? v[k][i] * r * w[i] : v[k][i];
                    store8(dst + e, y, a.vec_rows);
                }
            }
        }
    }
    __syncthreads();
    if (dst && lane < half / 8) {
        Turn8<T> r;
        r.load(x + a.rank, a.rot, lane, a.interleaved, a.vec_latent);
        r.store(dst + a.rank, cs[warp], a.rot, lane, a.interleaved, a.vec_rows);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if ((int)threadIdx.x + j * kRowThreads < parts) put(ahead[j], threadIdx.x + j * kRowThreads);
    for (int i = threadIdx.x + kAhead * kRowThreads; i < parts; i += kRowThreads) {
        Turn8<T> x;
        fetch(x, i);
        put(x, i);
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
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0 && threadIdx.x == 0) seq_lens[b] = min(L_max, L + 1 + acc);
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
    a.tokens = (long long)B * N >= 4096 ? mcsd::kRowTokens : 1;
    const dim3 grid((N + a.tokens - 1) / a.tokens, B);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == MCSD_F32) mcsd::latent_rows_kernel<float><<<grid, mcsd::kRowThreads, 0, s>>>(a);
    else mcsd::latent_rows_kernel<__nv_bfloat16><<<grid, mcsd::kRowThreads, 0, s>>>(a);
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
