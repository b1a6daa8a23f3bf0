// From a target layer's projections to what tree attention takes: RMS norm of every query and key head, rotation by the
// token's position (prefix length + depth in the tree; mcsd_build_mask hands out the depths), and the change from
// token-major to head-major rows, in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          (skipped without a weight)
//   angle = position * freq[i];   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin)   for every rotated pair (a, b)
//
// Every element is read once and written once, so memory bounds it (launch latency for single tokens).  A group of
// D / 8 lanes holds one head, eight consecutive elements per lane: 16-byte loads and stores for bf16, the sum of squares
// by shuffles inside the group, and for pairs that lie half a rotation apart the other element from the lane that has
// it.  The angles of a token are the same for all heads: a block works on one or a few whole tokens, its threads first reduce
// position * freq / 2 pi to a fraction of a turn in 64 bits (a far position has no bits left for the angle in 32) and
// leave sine and cosine in shared memory while the first head rows are on their way.
#include "norm_rope.cuh"

namespace mcsd {

constexpr int kRopeThreads = 256;

template <typename T> struct Row8;
template <> struct Row8<__nv_bfloat16> {
    __device__ __forceinline__ static void load(const __nv_bfloat16* p, float (&x)[8]) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ static void store(__nv_bfloat16* p, const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ static float one(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ __forceinline__ static __nv_bfloat16 back(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Row8<float> {
    __device__ __forceinline__ static void load(const float* p, float (&x)[8]) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ static void store(float* p, const float (&x)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
    __device__ __forceinline__ static float one(float v) { return v; }
    __device__ __forceinline__ static float back(float v) { return v; }
};
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    if (VEC) {
        Row8<T>::load(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = Row8<T>::one(p[e]);
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    if (VEC) {
        Row8<T>::store(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = Row8<T>::back(x[e]);
    }
}

// grid: (groups of TOK tokens, head splits).  VEC: every row starts on a 16-byte boundary.
template <typename T, int D, bool VEC, int TOK>
__global__ void __launch_bounds__(kRopeThreads, 3)
qk_norm_rope_kernel(const NormRopeArgs a) {
    constexpr int LPH = D / 8;                                // lanes per head
    constexpr int HPB = kRopeThreads / LPH;                   // heads of a block at a time
    constexpr int U = 3;                                      // of them whose loads are in flight together
    __shared__ float2 s_cs[TOK][D / 2];
    const int tid = threadIdx.x, c = tid % LPH;
    const int half = a.rot_dim >> 1;
    const int H_all = a.H_q + 2 * a.H_kv, H_qk = a.H_q + a.H_kv;
    const long long token0 = (long long)blockIdx.x * TOK, tokens = (long long)a.B * a.N;
    // The rows of the block in the order (token, head), `per` heads to a token; this thread takes every HPB-th.
    const int per = (H_all + gridDim.y - 1) / gridDim.y, h_lo = blockIdx.y * per;
    const int rows = per * TOK;

    struct Row { const T* from; T* to; int h, tok; };          // h < 0: nothing there
    auto row_at = [&](int i) -> Row {
        Row x;
        x.tok = TOK == 1 ? 0 : i / per;
        x.h = h_lo + i - x.tok * per;
        const long long token = token0 + x.tok;
        if (i >= rows || x.h >= H_all || token >= tokens) { x.h = -1; return x; }
        const int b = (int)(token / a.N), n = (int)(token - (long long)b * a.N);
        if (a.n_active && n >= a.n_active[b]) { x.h = -1; return x; }
        const size_t N = a.N;
        if (x.h < a.H_q) {
            x.from = static_cast<const T*>(a.q_in) + b * a.q_batch + n * a.q_token + (long long)x.h * D;
            x.to = static_cast<T*>(a.q_out) + (((size_t)b * a.H_q + x.h) * N + n) * D;
        } else if (x.h < H_qk) {
            x.from = static_cast<const T*>(a.k_in) + b * a.k_batch + n * a.k_token + (long long)(x.h - a.H_q) * D;
            x.to = static_cast<T*>(a.k_out) + (((size_t)b * a.H_kv + (x.h - a.H_q)) * N + n) * D;
        } else {
            x.from = static_cast<const T*>(a.v_in) + b * a.v_batch + n * a.v_token + (long long)(x.h - H_qk) * D;
            x.to = static_cast<T*>(a.v_out) + (((size_t)b * a.H_kv + (x.h - H_qk)) * N + n) * D;
        }
        return x;
    };

    float x[U][8];
    Row at[U];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = row_at(i0 + u * HPB);
            if (at[u].h >= 0) load8<T, VEC>(at[u].from + 8 * c, x[u]);
        }
    };
    const int i_first = tid / LPH;
    fetch(i_first);
    for (int i = tid; i < TOK * half; i += kRopeThreads) {
        const int tok = i / half, j = i - tok * half;
        const long long token = token0 + tok;
        if (token < tokens) {
            const int b = (int)(token / a.N), n = (int)(token - (long long)b * a.N);
            const long long pos = (long long)a.seq_lens[b] + (a.depth ? a.depth[n] : n);
            double turn = (double)pos * a.freqs[j] * 0.15915494309189533577;    // 1 / (2 pi)
            turn -= rint(turn);
            float sn, cs;
            sincospif(2.0f * (float)turn, &sn, &cs);
            s_cs[tok][j] = make_float2(cs, sn);
        }
    }
    __syncthreads();
    // the loop runs alike for all lanes of a warp (shuffles), whatever heads they hold
    for (int i0 = 0; i0 < rows; i0 += U * HPB) {
        if (i0 > 0) fetch(i0 + i_first);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = at[u].h;
            const bool is_q = h >= 0 && h < a.H_q, is_k = h >= a.H_q && h < H_qk;
            const float2* const cs_of = s_cs[at[u].tok < TOK ? at[u].tok : 0];
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = h >= 0 ? x[u][e] : 0.f;
            if (a.q_weight || a.k_weight) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(y[e], y[e], sum);
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float inv = rsqrtf(sum * (1.0f / D) + a.eps);
                const void* const weight = is_q ? a.q_weight : is_k ? a.k_weight : nullptr;
                if (weight) {
                    float w[8];
                    load8<T, VEC>(static_cast<const T*>(weight) + 8 * c, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= inv * w[e];
                }
            }
            if (a.interleaved) {
                if (is_q || is_k) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const int i = 4 * c + e / 2;
                        if (i < half) {
                            const float2 cs = cs_of[i];
                            const float y0 = y[e], y1 = y[e + 1];
                            y[e] = y0 * cs.x - y1 * cs.y;
                            y[e + 1] = y1 * cs.x + y0 * cs.y;
                        }
                    }
                }
            } else if (half > 0) {
                // element i pairs with i + half, which lies half / 8 lanes further on (half is a multiple of 8)
                const int apart = half >> 3;
                const bool low = c < apart, high = !low && c < 2 * apart;
                const int from = (tid & 31) + (low ? apart : high ? -apart : 0);
                float z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = __shfl_sync(0xffffffffu, y[e], from);
                if ((is_q || is_k) && (low || high)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 cs = cs_of[8 * (low ? c : c - apart) + e];
                        y[e] = low ? y[e] * cs.x - z[e] * cs.y : y[e] * cs.x + z[e] * cs.y;
                    }
                }
            }
            if (h >= 0) store8<T, VEC>(at[u].to + 8 * c, y);
        }
    }
}

template <typename T, int D>
static int launch(const NormRopeArgs& a, bool vec, cudaStream_t stream) {
    constexpr int HPB = kRopeThreads / (D / 8);
    const int H_all = a.H_q + 2 * a.H_kv;
    const long long tokens = (long long)a.B * a.N;
    // With few tokens the heads of a token go to several blocks (each repeats the token's angles); with many, a block takes
    // four whole tokens, whose angles keep all its threads busy once.
    const bool many = tokens >= 4 * 296;
    const dim3 grid((unsigned)(many ? (tokens + 3) / 4 : tokens), (unsigned)(tokens < 296 ? (H_all + HPB - 1) / HPB : 1));
    if (many && vec) qk_norm_rope_kernel<T, D, true, 4><<<grid, kRopeThreads, 0, stream>>>(a);
    else if (many) qk_norm_rope_kernel<T, D, false, 4><<<grid, kRopeThreads, 0, stream>>>(a);
    else if (vec) qk_norm_rope_kernel<T, D, true, 1><<<grid, kRopeThreads, 0, stream>>>(a);
    else qk_norm_rope_kernel<T, D, false, 1><<<grid, kRopeThreads, 0, stream>>>(a);
    MCSD_CUDA_CHECK(cudaGetLastError());
    count_launches(1);
    return MCSD_OK;
}

}  // namespace mcsd

extern "C" int mcsd_qk_norm_rope(const void* q_in, const void* k_in, const void* v_in, const int64_t* strides, const void* q_weight,
                                 const void* k_weight, float eps, const double* freqs, int rot_dim, int interleaved,
                                 const int32_t* seq_lens, const int32_t* depth, const int32_t* n_active, void* q_out, void* k_out,
                                 void* v_out, int B, int H_q, int H_kv, int N, int D, int dtype, void* stream) {
    if (!q_in || !k_in || !v_in || !strides || !seq_lens || !q_out || !k_out || !v_out || (rot_dim > 0 && !freqs)) return MCSD_ERR_NULL;
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (B < 1 || N < 1 || H_q < 1 || H_kv < 1 || (D != 64 && D != 128) || H_q > 65535 || H_kv > 65535) return MCSD_ERR_BAD_SHAPE;
    if ((long long)B * N > 0x7FFFFFFFLL) return MCSD_ERR_BAD_SHAPE;
    if (rot_dim < 0 || rot_dim > D || rot_dim % 2 != 0 || (!interleaved && rot_dim % 16 != 0)) return MCSD_ERR_BAD_SHAPE;
    if (!(eps >= 0.f)) return MCSD_ERR_BAD_SHAPE;
    mcsd::NormRopeArgs a{q_in, k_in, v_in, strides[0], strides[1], strides[2], strides[3], strides[4], strides[5],
                         q_weight, k_weight, eps, freqs, rot_dim, interleaved != 0, seq_lens, depth, n_active,
                         q_out, k_out, v_out, B, H_q, H_kv, N};
    const int per16 = dtype == MCSD_BF16 ? 8 : 4;
    bool vec = true;
    for (const void* p : {q_in, k_in, v_in, static_cast<const void*>(q_out), static_cast<const void*>(k_out), static_cast<const void*>(v_out), q_weight, k_weight})
        vec = vec && (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
    for (int i = 0; i < 6; ++i) vec = vec && strides[i] % per16 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == MCSD_F32) return D == 64 ? mcsd::launch<float, 64>(a, vec, s) : mcsd::launch<float, 128>(a, vec, s);
    return D == 64 ? mcsd::launch<__nv_bfloat16, 64>(a, vec, s) : mcsd::launch<__nv_bfloat16, 128>(a, vec, s);
}
