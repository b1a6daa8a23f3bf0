// Rows into and out of the 4-bit prefix cache (page layout in kv4.cuh): append (a prompt's rows), commit (Fig. 1 step 6
// of the paper: the accepted tree rows of every layer) and read back.
//
// A row x of one head is held as   lo, hi = min x, max x;   s = bf16((hi - lo) / 15);   o = bf16(lo - 16 s);
// code = clamp(round_half_even((x - o) / s) - 16, 0, 15), 0 where s = 0;   value = s (16 + code) + o.
// The offset is rounded to nearest: it moves the levels by at most 2^-9 |o|, a fraction of a step for rows whose
// range is not small against their magnitude, and no more than the rounding of bf16 rows themselves otherwise.
//
// All three move bytes and little else.  A thread block owns a whole page while it writes: two rows share a byte of the
// value codes, so a page that is written in part is read, merged and written back by the one thread that owns a
// channel; no two blocks of a call touch the same page.
#include <type_traits>

#include "kv4.cuh"

namespace mcsd {

constexpr int kStoreThreads = 128;
constexpr int kStoreWarps = kStoreThreads / 32;

__device__ __forceinline__ float warp_min(float v) {
    float r;
    asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// The type that decides between two codes.  For bf16 rows x - o is a short number and fp32 division cannot turn a value
// next to the middle of two levels into the middle itself; fp32 rows have all 24 bits, so they are decided in 64.
template <typename T> struct Decide { using type = float; };
template <> struct Decide<float> { using type = double; };

__device__ __forceinline__ float div_ieee(float a, float b) { return __fdiv_rn(a, b); }
__device__ __forceinline__ double div_ieee(double a, double b) { return __ddiv_rn(a, b); }
__device__ __forceinline__ double round_even(double a) { return rint(a); }
__device__ __forceinline__ float round_even(float a) { return rintf(a); }
__device__ __forceinline__ __nv_bfloat16 to_bf16(float a) { return __float2bfloat16_rn(a); }
__device__ __forceinline__ __nv_bfloat16 to_bf16(double a) { return __float2bfloat16_rn((float)a); }   // by way of fp32 in both forms

// E consecutive elements as fp32; VEC: the address is a multiple of their size
template <int E, bool VEC> __device__ __forceinline__ void load_row(const float* p, float (&x)[E]) {
    if (VEC && E == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x; x[1] = v.y; x[E - 2] = v.z; x[E - 1] = v.w;
    } else if (VEC) {
        const float2 v = *reinterpret_cast<const float2*>(p);
        x[0] = v.x; x[1] = v.y;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = p[e];
    }
}
template <int E, bool VEC> __device__ __forceinline__ void load_row(const __nv_bfloat16* p, float (&x)[E]) {
    if (VEC) {
        uint32_t w[E / 2];
        if (E == 4) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x; w[E / 2 - 1] = v.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = __bfloat162float(p[e]);
    }
}

// Codes of the E channels of one lane (a warp holds a row); returns the row's scale and offset.
template <typename T, int E>
__device__ __forceinline__ void quantise_row(const float (&x)[E], uint32_t (&code)[E], __nv_bfloat16& scale, __nv_bfloat16& offset) {
    using F = typename Decide<T>::type;
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < E; ++e) { lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]); }
    lo = warp_min(lo) + 0.f;                                  // rows of zeros: one bit pattern whatever their signs
    hi = warp_max(hi) + 0.f;
    scale = to_bf16(div_ieee((F)hi - (F)lo, (F)15));
    const F s = (F)__bfloat162float(scale);
    offset = to_bf16((F)lo - (F)16 * s);                      // 16 s is exact: the difference is rounded once either way
    const F o = (F)__bfloat162float(offset);
    if (sizeof(F) == 4 && (float)s > 1e-30f && (float)s < 1e30f) {
        // The quotient by the row's reciprocal, corrected once by its own remainder (which the fused multiply-add gives without
        // rounding): a value in the middle between two levels comes out as that middle, and no other value does.  Clamped
        // to 16..31, the sum with 1.5 2^23 rounds it to the nearest whole number, ties to even, whose low four bits are the code.
        const float r = 1.0f / (float)s;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = x[e] - (float)o, q0 = d * r, q = fmaf(fmaf(-q0, (float)s, d), r, q0);
            code[e] = __float_as_uint(fminf(fmaxf(q, 16.f), 31.f) + 12582912.f) & 15u;      // (a NaN counts as 16)
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const F t = round_even(div_ieee((F)x[e] - o, s));
        // comparisons are false for NaN (rows that are not finite): code 0
        const F c = t > (F)16 ? (t < (F)31 ? t : (F)31) : (F)16;
        code[e] = s > (F)0 ? (uint32_t)(int)c - 16u : 0u;
    }
}

template <int D>
struct PageSmem {
    alignas(16) unsigned char codes[kPageRows][D];   // value codes by row, one byte each
    uint32_t present;                         // rows of the page that are written
};

// Writes rows r0 .. r1 - 1 of a page; row_of(values, r) gives the source of page row r, or NULL to leave the row alone.
// Called by all threads of the block.
template <typename T, int D, bool VEC, typename RowOf>
__device__ __forceinline__ void store_page(unsigned char* page, int r0, int r1, PageSmem<D>& sm, RowOf row_of) {
    constexpr int E = D / 32;                                 // channels per lane
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __nv_bfloat16* scales = reinterpret_cast<__nv_bfloat16*>(page + kv4_scales_at(D));
    if (tid == 0) sm.present = 0;
    // what a page that is written in part keeps; on its way while the rows are made
    uint4* const dst = reinterpret_cast<uint4*>(page + kv4_values_at(D) + (tid < D ? tid : 0) * 16);
    const bool part = r0 > 0 || r1 < kPageRows;
    uint4 old = part && r0 < r1 ? *dst : make_uint4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll 4
    for (int r = r0 + warp; r < r1; r += kStoreWarps) {
        const T* ks = row_of(false, r);
        const T* vs = row_of(true, r);
        if (ks == nullptr || vs == nullptr) continue;         // uniform in the warp
        float xk[E], xv[E];
        load_row<E, VEC>(ks + lane * E, xk);
        load_row<E, VEC>(vs + lane * E, xv);
        uint32_t ck[E], cv[E];
        __nv_bfloat16 sk, ok, sv, ov;
        quantise_row<T, E>(xk, ck, sk, ok);
        quantise_row<T, E>(xv, cv, sv, ov);
        // keys: the 8 / E lanes of a word put their nibbles together
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) word |= ck[e] << kv4_bit((lane * E + e) & 7);
#pragma unroll
        for (int o = 1; o < 8 / E; o <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, o);
        const int w = lane * E / 8;                           // word of the row
        if ((lane * E) % 8 == 0)
            *reinterpret_cast<uint32_t*>(page + (size_t)(w >> 2) * (kPageRows * 16) + r * 16 + (w & 3) * 4) = word;
        if (E == 4) *reinterpret_cast<uint32_t*>(&sm.codes[r][lane * E]) = cv[0] | (cv[1] << 8) | (cv[E - 2] << 16) | (cv[E - 1] << 24);
        else *reinterpret_cast<unsigned short*>(&sm.codes[r][lane * E]) = (unsigned short)(cv[0] | (cv[1] << 8));
        if (lane == 0) {
            scales[r] = sk;
            scales[kPageRows + r] = ok;
            scales[2 * kPageRows + r] = sv;
            scales[3 * kPageRows + r] = ov;
            atomicOr(&sm.present, 1u << r);
        }
    }
    __syncthreads();
    const uint32_t present = sm.present;
    if (tid < D && present != 0) {
        uint32_t w[4] = {0, 0, 0, 0};
        if (present == 0xFFFFFFFFu) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[j] |= (uint32_t)sm.codes[8 * j + e][tid] << kv4_bit(e);
        } else {
            if (!part) old = *dst;                            // a whole page of which a row is left out (a malformed node)
            const uint32_t keep[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = 8 * j + e;
                    w[j] |= (present >> r) & 1u ? (uint32_t)sm.codes[r][tid] << kv4_bit(e) : keep[j] & (0xFu << kv4_bit(e));
                }
        }
        *dst = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncthreads();                                          // the codes may be overwritten
}

// grid: (pages that T rows can touch, B * H)
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kStoreThreads)
append_kv4_kernel(const T* __restrict__ k, const T* __restrict__ v, unsigned char* __restrict__ cache,
                  const int32_t* __restrict__ start, const int32_t* __restrict__ n_new, int H, int T_rows, int pages) {
    __shared__ PageSmem<D> sm;
    const int bh = blockIdx.y, b = bh / H;
    const int first = start[b], n = n_new ? min(max(n_new[b], 0), T_rows) : T_rows;
    if (first < 0) return;
    const long long page = (long long)(first / kPageRows) + blockIdx.x;
    const long long row0 = page * kPageRows;                  // cache row of the page's row 0
    if (page >= pages || row0 >= (long long)first + n) return;
    const int r0 = (int)max((long long)first - row0, 0LL), r1 = (int)min((long long)first + n - row0, (long long)kPageRows);
    const size_t src = (size_t)bh * T_rows;
    store_page<T, D, VEC>(cache + ((size_t)bh * pages + page) * kv4_page_bytes(D), r0, r1, sm, [&](bool values, int r) {
        return (values ? v : k) + (src + (size_t)(row0 + r - first)) * D;
    });
}

// grid: (B * H, n_layers)
template <typename T, int D>
__global__ void __launch_bounds__(kStoreThreads)
commit_kv4_kernel(void* const* __restrict__ cache_layers, const void* const* __restrict__ k_tree_layers,
                  const void* const* __restrict__ v_tree_layers, const int32_t* __restrict__ seq_lens,
                  const int32_t* __restrict__ accept_len, const int32_t* __restrict__ out_nodes,
                  const int32_t* __restrict__ best_root, int n_levels, int H, int N, int pages) {
    __shared__ PageSmem<D> sm;
    const int bh = blockIdx.x, b = bh / H, layer = blockIdx.y;
    const int L_max = pages * kPageRows;
    const int L = min(max(seq_lens[b], 0), L_max);
    const int acc = min(max(accept_len[b], 0), n_levels);
    const int end = min(L + 1 + acc, L_max);                  // rows beyond the cache are dropped
    const T* kt = static_cast<const T*>(k_tree_layers[layer]) + (size_t)bh * N * D;
    const T* vt = static_cast<const T*>(v_tree_layers[layer]) + (size_t)bh * N * D;
    unsigned char* head = static_cast<unsigned char*>(cache_layers[layer]) + (size_t)bh * pages * kv4_page_bytes(D);
    // (the pointers come from a table on the device, so their alignment is only known here)
    const bool vec = ((reinterpret_cast<uintptr_t>(kt) | reinterpret_cast<uintptr_t>(vt)) & 15u) == 0;
    for (int page = L / kPageRows; page * kPageRows < end; ++page) {
        const int row0 = page * kPageRows;
        auto row_of = [&](bool values, int r) -> const T* {
            const int i = row0 + r - L;                       // 0: the winning root, else accepted node i - 1
            const int node = i == 0 ? best_root[b] : out_nodes[(size_t)b * n_levels + (i - 1)];
            if (node < 0 || node >= N) return nullptr;        // malformed verify output: leave the row alone
            return (values ? vt : kt) + (size_t)node * D;
        };
        unsigned char* const at = head + (size_t)page * kv4_page_bytes(D);
        if (vec) store_page<T, D, true>(at, max(L - row0, 0), min(end - row0, kPageRows), sm, row_of);
        else store_page<T, D, false>(at, max(L - row0, 0), min(end - row0, kPageRows), sm, row_of);
    }
}

__global__ void grow_lens_kernel(int32_t* __restrict__ seq_lens, const int32_t* __restrict__ accept_len, int n_levels, int B, int L_max) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= B) return;
    const int L = min(max(seq_lens[b], 0), L_max);
    seq_lens[b] = min(L_max, L + 1 + min(max(accept_len[b], 0), n_levels));
}

template <typename T> __device__ __forceinline__ T store_as(float v);
template <> __device__ __forceinline__ float store_as<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 store_as<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// eight values as a row piece of T
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// grid: (pages that T rows can touch, B * H, n_layers); a block turns the rows of one page into rows of k and v.  Both are
// written as pieces of eight channels; the codes of a row's values are put side by side in shared memory first.  VEC: k and
// v are 16-byte aligned.
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kStoreThreads)
read_kv4_kernel(const void* const* __restrict__ cache_layers, const int32_t* __restrict__ first_rows, const int32_t* __restrict__ n_rows,
                int H, int T_rows, int pages, T* __restrict__ k, T* __restrict__ v) {
    __shared__ PageSmem<D> sm;
    const int bh = blockIdx.y, b = bh / H, layer = blockIdx.z, tid = threadIdx.x;
    const long long first = first_rows[b];
    const int n = n_rows ? min(max(n_rows[b], 0), T_rows) : T_rows;
    const long long page = (first >= 0 ? first / kPageRows : -((-first + kPageRows - 1) / kPageRows)) + blockIdx.x;
    const long long row0 = page * kPageRows;                  // the page's rows are rows row0 - first .. of k and v
    const int r0 = (int)max(first - row0, 0LL), r1 = (int)min(first + T_rows - row0, (long long)kPageRows);
    if (r0 >= r1) return;
    const bool there = page >= 0 && page < pages;
    const unsigned char* at = static_cast<const unsigned char*>(cache_layers[layer]) + ((size_t)bh * pages + (there ? page : 0)) * kv4_page_bytes(D);
    const __nv_bfloat16* sc = reinterpret_cast<const __nv_bfloat16*>(at + kv4_scales_at(D));
    const size_t out0 = ((size_t)layer * gridDim.y + bh) * T_rows;
    if (there && tid < D) {
        const uint4 x = *reinterpret_cast<const uint4*>(at + kv4_values_at(D) + tid * 16);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int r = 0; r < kPageRows; ++r) sm.codes[r][tid] = (unsigned char)((w[r >> 3] >> kv4_bit(r & 7)) & 15u);
    }
    __syncthreads();
    for (int i = tid; i < (r1 - r0) * (D / 8); i += kStoreThreads) {
        const int r = r0 + i / (D / 8), c = i % (D / 8);
        const int t = (int)(row0 + r - first);
        float xk[8], xv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) xk[e] = xv[e] = 0.f;
        if (there && t < n) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(at + (size_t)(c >> 2) * (kPageRows * 16) + r * 16 + (c & 3) * 4);
            const uint2 u = *reinterpret_cast<const uint2*>(&sm.codes[r][8 * c]);
            const float ks = __bfloat162float(sc[r]), ko = __bfloat162float(sc[kPageRows + r]);
            const float vs = __bfloat162float(sc[2 * kPageRows + r]), vo = __bfloat162float(sc[3 * kPageRows + r]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xk[e] = kv4_value((w >> kv4_bit(e)) & 15u, ks, ko);
                xv[e] = kv4_value(((e < 4 ? u.x : u.y) >> (8 * (e & 3))) & 15u, vs, vo);
            }
        }
        T* const dk = k + (out0 + t) * D + 8 * c;
        T* const dv = v + (out0 + t) * D + 8 * c;
        if (VEC) {
            store8(dk, xk);
            store8(dv, xv);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { dk[e] = store_as<T>(xk[e]); dv[e] = store_as<T>(xv[e]); }
        }
    }
}

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The sizes all entry points of the 4-bit cache share.
static int check_cache(int B, int H, int D, int L_max, int dtype) {
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (B < 1 || H < 1 || (D != 64 && D != 128) || (long long)B * H > 65535) return MCSD_ERR_BAD_SHAPE;
    if (L_max < kPageRows || L_max % kPageRows != 0) return MCSD_ERR_BAD_SHAPE;
    return MCSD_OK;
}

// Calls f with the element type and head width of the call as template arguments.
template <typename F>
static int by_type(int dtype, int D, F f) {
    if (dtype == MCSD_F32) return D == 64 ? f(float{}, std::integral_constant<int, 64>{}) : f(float{}, std::integral_constant<int, 128>{});
    return D == 64 ? f(__nv_bfloat16{}, std::integral_constant<int, 64>{}) : f(__nv_bfloat16{}, std::integral_constant<int, 128>{});
}

}  // namespace mcsd

using namespace mcsd;

extern "C" size_t mcsd_kv4_cache_bytes(int B, int H, int D, int L_max) {
    if (check_cache(B, H, D, L_max, MCSD_BF16) != MCSD_OK) return 0;
    return (size_t)B * H * (L_max / kPageRows) * kv4_page_bytes(D);
}

extern "C" int mcsd_append_kv4(const void* k, const void* v, void* cache, const int32_t* start, const int32_t* n_new, int B,
                               int H, int T, int D, int L_max, int dtype, void* stream) {
    if (!k || !v || !cache || !start) return MCSD_ERR_NULL;
    const int st = check_cache(B, H, D, L_max, dtype);
    if (st != MCSD_OK) return st;
    if (T < 1 || !aligned16(cache)) return MCSD_ERR_BAD_SHAPE;
    const int pages = L_max / kPageRows;
    const long long touched = ((long long)T + kPageRows - 1) / kPageRows + 1;
    return by_type(dtype, D, [&](auto t, auto d) {
        using T_ = decltype(t);
        constexpr int D_ = decltype(d)::value;
        const dim3 grid((unsigned)(touched < pages ? touched : pages), (unsigned)(B * H));
        const bool vec = aligned16(k) && aligned16(v);         // rows are multiples of 16 bytes long
        auto* const kernel = vec ? append_kv4_kernel<T_, D_, true> : append_kv4_kernel<T_, D_, false>;
        kernel<<<grid, kStoreThreads, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<const T_*>(k), static_cast<const T_*>(v),
                                                                              static_cast<unsigned char*>(cache), start, n_new, H, T, pages);
        MCSD_CUDA_CHECK(cudaGetLastError());
        count_launches(1);
        return MCSD_OK;
    });
}

extern "C" int mcsd_read_kv4(const void* const* cache_layers, int n_layers, const int32_t* first, const int32_t* n_rows, int B,
                             int H, int T, int D, int L_max, int dtype, void* k, void* v, void* stream) {
    if (!cache_layers || !first || !k || !v) return MCSD_ERR_NULL;
    const int st = check_cache(B, H, D, L_max, dtype);
    if (st != MCSD_OK) return st;
    if (T < 1 || n_layers < 1 || n_layers > 65535) return MCSD_ERR_BAD_SHAPE;
    return by_type(dtype, D, [&](auto t, auto d) {
        using T_ = decltype(t);
        constexpr int D_ = decltype(d)::value;
        const dim3 grid((unsigned)(((long long)T + kPageRows - 1) / kPageRows + 1), (unsigned)(B * H), (unsigned)n_layers);
        auto* const kernel = aligned16(k) && aligned16(v) ? read_kv4_kernel<T_, D_, true> : read_kv4_kernel<T_, D_, false>;
        kernel<<<grid, kStoreThreads, 0, static_cast<cudaStream_t>(stream)>>>(
            cache_layers, first, n_rows, H, T, L_max / kPageRows, static_cast<T_*>(k), static_cast<T_*>(v));
        MCSD_CUDA_CHECK(cudaGetLastError());
        count_launches(1);
        return MCSD_OK;
    });
}

extern "C" int mcsd_commit_kv4(void* const* cache_layers, const void* const* k_tree_layers, const void* const* v_tree_layers,
                               int n_layers, int32_t* seq_lens, const int32_t* accept_len, const int32_t* out_nodes,
                               const int32_t* best_root, int n_levels, int B, int H, int N, int D, int L_max, int dtype, void* stream) {
    if (!cache_layers || !k_tree_layers || !v_tree_layers || !seq_lens || !accept_len || !out_nodes || !best_root) return MCSD_ERR_NULL;
    const int st = check_cache(B, H, D, L_max, dtype);
    if (st != MCSD_OK) return st;
    if (n_layers < 1 || n_layers > 65535 || N < 1 || N > MCSD_MAX_NODES || n_levels < 1 || n_levels > N) return MCSD_ERR_BAD_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return by_type(dtype, D, [&](auto t, auto d) {
        using T_ = decltype(t);
        constexpr int D_ = decltype(d)::value;
        commit_kv4_kernel<T_, D_><<<dim3((unsigned)(B * H), (unsigned)n_layers), kStoreThreads, 0, s>>>(
            cache_layers, k_tree_layers, v_tree_layers, seq_lens, accept_len, out_nodes, best_root, n_levels, H, N, L_max / kPageRows);
        MCSD_CUDA_CHECK(cudaGetLastError());
        grow_lens_kernel<<<(B + 127) / 128, 128, 0, s>>>(seq_lens, accept_len, n_levels, B, L_max);
        MCSD_CUDA_CHECK(cudaGetLastError());
        count_launches(2);
        return MCSD_OK;
    });
}
