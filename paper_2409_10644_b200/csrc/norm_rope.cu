// From a target layer's projections to what tree attention takes: RMS norm of every query and key head, rotation by the
// token's position (prefix length + depth in the tree; mcsd_build_mask hands out the depths), and the change from
// token-major to head-major rows, in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          (skipped without a weight)
//   angle = position * freq[i];   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin)   for every rotated pair (a, b)
//
// Every element is read once and written once, so memory bounds it (launch latency for single tokens).  To come near that
// bound the instructions per element have to be few: D / 8 lanes hold one head, and a lane takes four elements and the
// four they are rotated with, so that no pair crosses lanes (only the sum of squares does); it keeps one token's sines
// and cosines in registers for all the heads it works on, and the weights for all its rows; the arithmetic goes by two.
// The angles are reduced as position * freq / 2 pi to a fraction of a turn in 64 bits (a far position has no bits left
// for the angle in 32) by all threads of a block while the first rows are on their way.
//
// Measured: 8191 tokens of 48 heads of 128, norm and half rotated, bf16: 47 us, 4.3 TB/s of the 201 MB that have to move, with
// 69 % of the issue slots used by 5.5 warps per scheduler (77 registers: three blocks on a multiprocessor), so instructions
// bound it, not loads; 16 x 45 tokens of 96 heads: 10.2 us, 3.5 TB/s, 720 blocks where 444 run at a time, which
// spend much of their time at the barrier behind the angles; a single token 4.6 us, of which most is the launch.
#include "f32x2.cuh"
#include "norm_rope.cuh"

namespace mcsd {

constexpr int kRopeThreads = 256;

// four consecutive elements as they lie in memory; VEC: aligned to their size
template <typename T> struct Quad;
template <> struct Quad<__nv_bfloat16> {
    uint2 w;
    template <bool VEC> __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        if (VEC) {
            w = *reinterpret_cast<const uint2*>(p);
        } else {
            const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
            w = make_uint2(u[0] | ((uint32_t)u[1] << 16), u[2] | ((uint32_t)u[3] << 16));
        }
    }
    template <bool VEC> __device__ __forceinline__ void store(__nv_bfloat16* p) const {
        if (VEC) {
            *reinterpret_cast<uint2*>(p) = w;
        } else {
            unsigned short* u = reinterpret_cast<unsigned short*>(p);
            u[0] = (unsigned short)w.x; u[1] = (unsigned short)(w.x >> 16); u[2] = (unsigned short)w.y; u[3] = (unsigned short)(w.y >> 16);
        }
    }
    __device__ __forceinline__ void ones() { w = make_uint2(0x3F803F80u, 0x3F803F80u); }
    __device__ __forceinline__ void zero() { w = make_uint2(0u, 0u); }
    __device__ __forceinline__ float2 lo() const { return make_float2(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u)); }
    __device__ __forceinline__ float2 hi() const { return make_float2(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u)); }
    __device__ __forceinline__ void set(float2 a, float2 b) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(a.x, a.y), y = __floats2bfloat162_rn(b.x, b.y);
        w = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
    }
};
template <> struct Quad<float> {
    float4 w;
    template <bool VEC> __device__ __forceinline__ void load(const float* p) {
        if (VEC) w = *reinterpret_cast<const float4*>(p);
        else w = make_float4(p[0], p[1], p[2], p[3]);
    }
    template <bool VEC> __device__ __forceinline__ void store(float* p) const {
        if (VEC) {
            *reinterpret_cast<float4*>(p) = w;
        } else {
            p[0] = w.x; p[1] = w.y; p[2] = w.z; p[3] = w.w;
        }
    }
    __device__ __forceinline__ void ones() { w = make_float4(1.f, 1.f, 1.f, 1.f); }
    __device__ __forceinline__ void zero() { w = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float2 lo() const { return make_float2(w.x, w.y); }
    __device__ __forceinline__ float2 hi() const { return make_float2(w.z, w.w); }
    __device__ __forceinline__ void set(float2 a, float2 b) { w = make_float4(a.x, a.y, b.x, b.y); }
};

// grid: groups of TOK tokens.  VEC: every row starts on a 16-byte boundary.
template <typename T, int D, bool VEC, int TOK>
__global__ void __launch_bounds__(kRopeThreads)
qk_norm_rope_kernel(const NormRopeArgs a) {
    constexpr int LPH = D / 8;                                // lanes per head
    constexpr int GPT = kRopeThreads / LPH / TOK;             // heads of one token at a time
    constexpr int U = sizeof(T) == 2 ? 4 : 2;                 // rows of a lane whose loads are in flight together
    __shared__ float4 s_cos[TOK][LPH], s_sin[TOK][LPH];
    const int tid = threadIdx.x, c = tid % LPH, group = tid / LPH, tok = group / GPT;
    const int half = a.rot_dim >> 1;
    const int H_all = a.H_q + 2 * a.H_kv, H_qk = a.H_q + a.H_kv;
    const long long token0 = (long long)blockIdx.x * TOK, tokens = (long long)a.B * a.N;
    const int h_first = group % GPT;
    const long long token = min(token0 + tok, tokens - 1);
    const int b = (int)(token / a.N), n = (int)(token - (long long)b * a.N);
    int h_end = H_all;
    if (token0 + tok >= tokens || (a.n_active && n >= a.n_active[b])) h_end = 0;    // the same for all lanes of a warp

    // Where this lane's two quads lie in a row.  Neighbours are pairs: eight elements in a row.  Pairs half a rotation apart:
    // elements 4c .. 4c + 3 and their partners; what is not rotated lies behind, and is split down its middle.
    const int off_a = a.interleaved ? 8 * c : 4 * c < half ? 4 * c : 4 * c + half;
    const int off_b = a.interleaved ? 8 * c + 4 : 4 * c < half ? 4 * c + half : 4 * c + D / 2;

    const T* const q_in = static_cast<const T*>(a.q_in) + b * a.q_batch + n * a.q_token;
    const T* const k_in = static_cast<const T*>(a.k_in) + b * a.k_batch + n * a.k_token;
    const T* const v_in = static_cast<const T*>(a.v_in) + b * a.v_batch + n * a.v_token;
    Quad<T> xa[U], xb[U];
    auto fetch = [&](int h, int u) {
        xa[u].zero();
        xb[u].zero();
        if (h < h_end) {
            const T* const from = h < a.H_q ? q_in + (long long)h * D : h < H_qk ? k_in + (long long)(h - a.H_q) * D : v_in + (long long)(h - H_qk) * D;
            xa[u].template load<VEC>(from + off_a);
            xb[u].template load<VEC>(from + off_b);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(h_first + u * GPT, u);
    Quad<T> wqa, wqb, wka, wkb;
    wqa.ones(); wqb.ones(); wka.ones(); wkb.ones();
    if (a.q_weight) {
        wqa.template load<VEC>(static_cast<const T*>(a.q_weight) + off_a);
        wqb.template load<VEC>(static_cast<const T*>(a.q_weight) + off_b);
    }
    if (a.k_weight) {
        wka.template load<VEC>(static_cast<const T*>(a.k_weight) + off_a);
        wkb.template load<VEC>(static_cast<const T*>(a.k_weight) + off_b);
    }
    for (int i = tid; i < TOK * half; i += kRopeThreads) {
        const int t = i / half, j = i - t * half;
        if (token0 + t < tokens) {
            const int tb = (int)((token0 + t) / a.N), tn = (int)(token0 + t - (long long)tb * a.N);
            const long long pos = (long long)a.seq_lens[tb] + (a.depth ? a.depth[tn] : tn);
            double turn = (double)pos * a.freqs[j] * 0.15915494309189533577;    // 1 / (2 pi)
            turn -= rint(turn);
            float sn, cs;
            sincospif(2.0f * (float)turn, &sn, &cs);
            reinterpret_cast<float*>(s_cos[t])[j] = cs;
            reinterpret_cast<float*>(s_sin[t])[j] = sn;
        }
    }
    __syncthreads();
    const float4 cs = s_cos[tok][c], sn = s_sin[tok][c];      // of pairs 4c .. 4c + 3; not set, and not used, from `half` on
    const size_t N = a.N;
    T* const q_out = static_cast<T*>(a.q_out) + ((size_t)b * a.H_q * N + n) * D;
    T* const k_out = static_cast<T*>(a.k_out) + ((size_t)b * a.H_kv * N + n) * D;
    T* const v_out = static_cast<T*>(a.v_out) + ((size_t)b * a.H_kv * N + n) * D;
    const bool norms = a.q_weight || a.k_weight;
    // the loop runs alike for all lanes of a warp (shuffles), whatever heads they hold
    for (int h0 = h_first; h0 - h_first < H_all; h0 += U * GPT) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * GPT;
            const bool is_q = h < a.H_q, is_v = h >= H_qk;
            Quad<T> ya = xa[u], yb = xb[u];
            float2 a0 = ya.lo(), a1 = ya.hi(), b0 = yb.lo(), b1 = yb.hi();
            const Quad<T> va = ya, vb = yb;                   // values pass through unchanged
            fetch(h + U * GPT, u);
            if (norms) {
                float2 sq = mul_f32x2(a0, a0);
                sq = fma_f32x2(a1, a1, sq);
                sq = fma_f32x2(b0, b0, sq);
                sq = fma_f32x2(b1, b1, sq);
                float sum = sq.x + sq.y;
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float inv = (is_q ? a.q_weight : a.k_weight) ? rsqrtf(sum * (1.0f / D) + a.eps) : 1.0f;
                const float2 inv2 = make_float2(inv, inv);
                Quad<T> wa = wqa, wb = wqb;
                if (!is_q) { wa = wka; wb = wkb; }
                a0 = mul_f32x2(a0, mul_f32x2(wa.lo(), inv2));
                a1 = mul_f32x2(a1, mul_f32x2(wa.hi(), inv2));
                b0 = mul_f32x2(b0, mul_f32x2(wb.lo(), inv2));
                b1 = mul_f32x2(b1, mul_f32x2(wb.hi(), inv2));
            }
            if (a.interleaved) {
                auto turn = [&](float2& y, int pair, float co, float si) {
                    if (pair < half) y = make_float2(y.x * co - y.y * si, y.y * co + y.x * si);
                };
                turn(a0, 4 * c, cs.x, sn.x);
                turn(a1, 4 * c + 1, cs.y, sn.y);
                turn(b0, 4 * c + 2, cs.z, sn.z);
                turn(b1, 4 * c + 3, cs.w, sn.w);
            } else if (4 * c < half) {                        // half is a multiple of 8
                const float2 c0 = make_float2(cs.x, cs.y), c1 = make_float2(cs.z, cs.w), s0 = make_float2(sn.x, sn.y), s1 = make_float2(sn.z, sn.w);
                const float2 m0 = make_float2(-sn.x, -sn.y), m1 = make_float2(-sn.z, -sn.w);
                const float2 x0 = a0, x1 = a1;
                a0 = fma_f32x2(b0, m0, mul_f32x2(x0, c0));
                a1 = fma_f32x2(b1, m1, mul_f32x2(x1, c1));
                b0 = fma_f32x2(x0, s0, mul_f32x2(b0, c0));
                b1 = fma_f32x2(x1, s1, mul_f32x2(b1, c1));
            }
            ya.set(a0, a1);
            yb.set(b0, b1);
            if (is_v) { ya = va; yb = vb; }
            if (h < h_end) {
                T* const to = is_q ? q_out + (size_t)h * N * D : !is_v ? k_out + (size_t)(h - a.H_q) * N * D : v_out + (size_t)(h - H_qk) * N * D;
                ya.template store<VEC>(to + off_a);
                yb.template store<VEC>(to + off_b);
            }
        }
    }
}

template <typename T, int D>
static int launch(const NormRopeArgs& a, bool vec, cudaStream_t stream) {
    const long long tokens = (long long)a.B * a.N;
    // One block per token while there are few; from 1184 tokens on (eight for each of the 148 multiprocessors, which hold three
    // blocks each) a block takes four, whose angles keep all its threads busy once.  8191 tokens: 47 us against 70 us with
    // a block each; 720 tokens: 12.4 us with a block each against 14.1 us by fours.
    const bool many = tokens >= 8 * 148;
    if (!vec) qk_norm_rope_kernel<T, D, false, 1><<<(unsigned)tokens, kRopeThreads, 0, stream>>>(a);
    else if (many) qk_norm_rope_kernel<T, D, true, 4><<<(unsigned)((tokens + 3) / 4), kRopeThreads, 0, stream>>>(a);
    else qk_norm_rope_kernel<T, D, true, 1><<<(unsigned)tokens, kRopeThreads, 0, stream>>>(a);
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
