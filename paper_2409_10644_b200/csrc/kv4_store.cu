// Rows into and out of the 4-bit prefix cache (page layout in kv4.cuh): append (a prompt's rows), commit (Fig. 1 step 6
// of the paper: the accepted tree rows of every layer) and read back.
//
// A row x of one head is held as   lo, hi = min x, max x;   s = bf16((hi - lo) / 15);   o = bf16(lo - 16 s);
// code = clamp(round_half_even((x - o) / s) - 16, 0, 15), 0 where s = 0;   value = s (16 + code) + o.
// The offset is rounded to nearest: it moves the levels by at most 2^-9 |o|, a fraction of a step for rows whose
// range is not small against their magnitude, and no more than the rounding of bf16 rows themselves otherwise.
//
// All three move bytes and little else; what bounds them is how many instructions they spend on an element.
// A warp turns eight rows, the ones that share the 32-bit words of the value codes, into codes: their loads are in flight
// together, the scales and offsets of all of them are computed at once (one lane per row), and every code is added to its
// words as it is made.  Two rows share a byte of the value codes: one warp owns all of its words, and where only some of
// the rows are written it merges with what is there; no two warps of a call touch the same word.
//
// Measured with heads of 128 in bf16: 8191 rows of 32 heads appended in 52 us (170 MB, 3.3 TB/s; 69 % of the issue slots at 4.7
// warps per scheduler) and read back in 35 us (4.9 TB/s; 64 % at 8.9); rows accepted by 16 sequences in 32 layers of 32 heads
// committed in 37 us (44 us without the branches over absent rows, which a page that is written whole does not want; 37 % of
// the slots, most of the rest waiting for a chain of three dependent loads for every one of 16384 heads) and read back
// in 35 us (71 %, in 32768 blocks, of which half find nothing to do).  Whole 32-byte sectors would let both go in 15 us.
#include <type_traits>

#include "f32x2.cuh"
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

__device__ __forceinline__ __nv_bfloat16 to_bf16(float a) { return __float2bfloat16_rn(a); }
__device__ __forceinline__ __nv_bfloat16 to_bf16(double a) { return __float2bfloat16_rn((float)a); }   // by way of fp32 in both forms

// E consecutive elements as they lie in memory; VEC: the address is a multiple of their size.  get() gives a neighbouring pair.
template <typename T, int E> struct Piece;
template <int E> struct Piece<float, E> {
    float x[E];
    template <bool VEC> __device__ __forceinline__ void load(const float* p) {
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
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
    }
    __device__ __forceinline__ float2 get(int e) const { return make_float2(x[e], x[e + 1]); }
};
template <int E> struct Piece<__nv_bfloat16, E> {
    uint32_t w[E / 2];
    template <bool VEC> __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        if (VEC && E == 4) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x; w[E / 2 - 1] = v.y;
        } else if (VEC) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
            for (int e = 0; e < E / 2; ++e) w[e] = u[2 * e] | ((uint32_t)u[2 * e + 1] << 16);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) w[e] = 0u;
    }
    __device__ __forceinline__ float2 get(int e) const {
        return make_float2(__uint_as_float(w[e / 2] << 16), __uint_as_float(w[e / 2] & 0xFFFF0000u));
    }
};

// What a row's codes are made from.  The quotient (x - o) / s is the product with the reciprocal of s, corrected once by its
// own remainder, which the fused multiply-add gives without rounding.  s has 8 significant bits, so no quotient is so
// close to the middle of two neighbouring numbers that this could round it otherwise than a division does: a value in
// the middle between two levels comes out as that middle, and no other value does.  bf16 rows are decided in 32 bits; fp32 rows,
// whose x - o has more bits than that, in 64.  s = 0, infinite or NaN gives 0 or NaN here, and a NaN counts as code 0.
//
// code_bits() returns kCodeBase + code: the quotient, clamped to 16 .. 31, plus 1.5 2^23 is rounded to the nearest whole
// number, ties to even, and its low bits are that number.
constexpr uint32_t kCodeBase = 0x4B400010u;
template <typename T> struct RowScale;
template <> struct RowScale<__nv_bfloat16> {
    using F = float;
    float2 minus_o, minus_s, r;
    __device__ __forceinline__ RowScale(float s, float o, float inv) : minus_o(make_float2(-o, -o)), minus_s(make_float2(-s, -s)), r(make_float2(inv, inv)) {}
    // Outside this range products with the reciprocal could lose bits or overflow, and the division is made instead.
    __device__ __forceinline__ static bool plain(float s) { return !(s > 0.f && s <= 1e-30f) && !(s >= 1e30f && s <= 3.4e38f); }
    __device__ __forceinline__ static float inverse(float s) { return s > 0.f ? 1.0f / s : 0.f; }
    template <bool PLAIN>
    __device__ __forceinline__ void code_bits(float2 x, uint32_t& c0, uint32_t& c1) const {
        const float2 d = add_f32x2(x, minus_o);
        float2 q;
        if (PLAIN) {
            const float2 q0 = mul_f32x2(d, r);
            q = fma_f32x2(fma_f32x2(q0, minus_s, d), r, q0);
        } else {
            q = make_float2(minus_s.x < 0.f ? __fdiv_rn(d.x, -minus_s.x) : 0.f, minus_s.y < 0.f ? __fdiv_rn(d.y, -minus_s.y) : 0.f);
        }
        q = add_f32x2(make_float2(fminf(fmaxf(q.x, 16.f), 31.f), fminf(fmaxf(q.y, 16.f), 31.f)), make_float2(12582912.f, 12582912.f));
        c0 = __float_as_uint(q.x);
        c1 = __float_as_uint(q.y);
    }
};
template <> struct RowScale<float> {
    using F = double;
    double s, o, r;
    __device__ __forceinline__ RowScale(float s_, float o_, float) : s(s_), o(o_), r(s_ > 0.f ? 1.0 / (double)s_ : 0.0) {}
    __device__ __forceinline__ static bool plain(float) { return true; }           // no fp32 number is near the limits of 64 bits
    __device__ __forceinline__ static float inverse(float) { return 0.f; }
    __device__ __forceinline__ uint32_t one(float x) const {
        const double d = (double)x - o, q0 = d * r, q = fma(fma(-q0, s, d), r, q0);
        return (uint32_t)__double2loint(fmin(fmax(q, 16.0), 31.0) + 6755399441055744.0) - 16u + kCodeBase;    // 1.5 2^52, likewise
    }
    template <bool PLAIN>
    __device__ __forceinline__ void code_bits(float2 x, uint32_t& c0, uint32_t& c1) const { c0 = one(x.x); c1 = one(x.y); }
};

constexpr int kGroup = 8;                                     // rows that share the words of the value codes

// Makes the codes of rows 8g .. 8g + 7 of a page as far as `present` has their bit; one whole warp.  k_row(r), v_row(r) give the
// sources.  Key codes, scales and offsets go to the page, the words of the value codes (channels E lane ..) to vw, 0 in
// the nibbles of absent rows.  SPARSE: few rows are expected, and the instructions for absent ones are branched over, else they
// are made as rows of zeros.
template <typename T, int D, bool VEC, bool SPARSE, typename KRow, typename VRow>
__device__ __forceinline__ void make_group(unsigned char* page, int g, uint32_t present, KRow k_row, VRow v_row, uint32_t (&vw)[D / 32]) {
    constexpr int E = D / 32;                                 // channels per lane
    using F = typename RowScale<T>::F;
    const int lane = threadIdx.x & 31;
    Piece<T, E> x[2][kGroup];
#pragma unroll
    for (int r = 0; r < kGroup; ++r) {
        x[0][r].zero();
        x[1][r].zero();
        if ((present >> r) & 1u) {
            x[0][r].template load<VEC>(k_row(r) + lane * E);
            x[1][r].template load<VEC>(v_row(r) + lane * E);
        }
    }
    // lane r keeps the range of key row r, lane 8 + r that of value row r
    float lo_mine = 0.f, hi_mine = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * kGroup; ++i) {
        if (SPARSE && ((present >> (i % kGroup)) & 1u) == 0u) continue;
        const Piece<T, E>& p = x[i / kGroup][i % kGroup];
        float2 lo = p.get(0), hi = lo;
        if (E == 4) {
            const float2 z = p.get(E - 2);
            lo = make_float2(fminf(lo.x, z.x), fminf(lo.y, z.y));
            hi = make_float2(fmaxf(hi.x, z.x), fmaxf(hi.y, z.y));
        }
        const float l = warp_min(fminf(lo.x, lo.y)), h = warp_max(fmaxf(hi.x, hi.y));
        if (lane == i) { lo_mine = l; hi_mine = h; }
    }
    lo_mine += 0.f;                                           // rows of zeros: one bit pattern whatever their signs
    hi_mine += 0.f;
    const __nv_bfloat16 scale = to_bf16(((F)hi_mine - (F)lo_mine) / (F)15);
    const F s_mine = (F)__bfloat162float(scale);
    const __nv_bfloat16 offset = to_bf16((F)lo_mine - (F)16 * s_mine);      // 16 s is exact: the difference is rounded once either way
    const float s32 = __bfloat162float(scale), o32 = __bfloat162float(offset), inv = RowScale<T>::inverse(s32);
    if (lane < 2 * kGroup && ((present >> (lane % kGroup)) & 1u)) {
        __nv_bfloat16* const at = reinterpret_cast<__nv_bfloat16*>(page + kv4_scales_at(D)) + (lane / kGroup) * 2 * kPageRows + g * kGroup + lane % kGroup;
        at[0] = scale;
        at[kPageRows] = offset;
    }
    const bool plain = __all_sync(0xffffffffu, RowScale<T>::plain(s32));

    uint32_t kw[kGroup], sum[E];
    constexpr uint32_t kAll = 0x11111111u * kCodeBase;        // what the bases of eight codes add up to, modulo 2^32
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = SPARSE ? 0u : 0u - kAll;
    auto codes = [&](auto plain_t) {
        constexpr bool kPlain = decltype(plain_t)::value;
#pragma unroll
        for (int r = 0; r < kGroup; ++r) {
            kw[r] = 0u;
            if (SPARSE && ((present >> r) & 1u) == 0u) continue;
            const RowScale<T> key(__shfl_sync(0xffffffffu, s32, r), __shfl_sync(0xffffffffu, o32, r), __shfl_sync(0xffffffffu, inv, r));
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                uint32_t c0, c1;
                key.template code_bits<kPlain>(x[0][r].get(e), c0, c1);
                kw[r] += ((c0 - kCodeBase) << kv4_bit(e)) + ((c1 - kCodeBase) << kv4_bit(e + 1));
            }
            const RowScale<T> val(__shfl_sync(0xffffffffu, s32, kGroup + r), __shfl_sync(0xffffffffu, o32, kGroup + r), __shfl_sync(0xffffffffu, inv, kGroup + r));
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                uint32_t c0, c1;
                val.template code_bits<kPlain>(x[1][r].get(e), c0, c1);
                sum[e] += (SPARSE ? c0 - kCodeBase : c0) << kv4_bit(r);
                sum[e + 1] += (SPARSE ? c1 - kCodeBase : c1) << kv4_bit(r);
            }
        }
    };
    if (plain) codes(std::true_type{});
    else codes(std::false_type{});
#pragma unroll
    for (int e = 0; e < E; ++e) vw[e] = sum[e];               // (rows of zeros have code 0)
    // The words of the key codes: the lanes of a word (2 or 4) put their nibbles together, even lanes for one row of a pair
    // of rows and odd lanes for the other.
    const int word = lane * E / 8, shift = lane * E % 8 * 2;  // elements lane E .. start at bit 2 (lane E mod 8)
#pragma unroll
    for (int r = 0; r < kGroup; r += 2) {
        if (SPARSE && ((present >> r) & 3u) == 0u) continue;
        const uint32_t w0 = kw[r] << shift, w1 = kw[r + 1] << shift;
        uint32_t w = (lane & 1 ? w1 : w0) | __shfl_xor_sync(0xffffffffu, lane & 1 ? w0 : w1, 1);
        if (E == 2) w |= __shfl_xor_sync(0xffffffffu, w, 2);
        const int row = r + (lane & 1);
        if (((present >> row) & 1u) && (E == 4 || (lane & 2) == 0))
            *reinterpret_cast<uint32_t*>(page + (word >> 2) * (kPageRows * 16) + (g * kGroup + row) * 16 + (word & 3) * 4) = w;
    }
}

// the nibbles of a word of value codes that belong to the rows of `present` (8 bits)
__device__ __forceinline__ uint32_t nibbles_of(uint32_t present) {
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < kGroup; ++r) m |= ((present >> r) & 1u) * (0xFu << kv4_bit(r));
    return m;
}

// grid: (pages that T rows can touch, B * H); warp g makes rows 8g .. 8g + 7 of the page
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kStoreThreads)
append_kv4_kernel(const T* __restrict__ k, const T* __restrict__ v, unsigned char* __restrict__ cache,
                  const int32_t* __restrict__ start, const int32_t* __restrict__ n_new, int H, int T_rows, int pages) {
    constexpr int E = D / 32;
    static_assert(kStoreWarps * kGroup == kPageRows, "one warp per group of rows");
    __shared__ alignas(16) uint32_t s_words[kStoreWarps][D];
    const int bh = blockIdx.y, b = bh / H, tid = threadIdx.x, lane = tid & 31, g = tid >> 5;
    const int first = start[b], n = n_new ? min(max(n_new[b], 0), T_rows) : T_rows;
    if (first < 0) return;
    const long long page = (long long)(first / kPageRows) + blockIdx.x;
    const long long row0 = page * kPageRows;                  // cache row of the page's row 0
    if (page >= pages || row0 >= (long long)first + n) return;
    const int r0 = (int)max((long long)first - row0, 0LL), r1 = (int)min((long long)first + n - row0, (long long)kPageRows);
    if (r0 >= r1) return;                                     // nothing to append, in the middle of a page
    unsigned char* const at = cache + ((size_t)bh * pages + page) * kv4_page_bytes(D);
    uint4* const dst = reinterpret_cast<uint4*>(at + kv4_values_at(D) + (tid < D ? tid : 0) * 16);
    uint4 old = make_uint4(0, 0, 0, 0);
    if (r0 > 0 || r1 < kPageRows) old = *dst;                 // what a page that is written in part keeps
    const uint32_t rows = (uint32_t)((1ULL << r1) - (1ULL << r0)), present = (rows >> (g * kGroup)) & 0xFFu;
    const long long src = (long long)bh * T_rows + (row0 + g * kGroup - first);   // row of k and v of the group's row 0
    uint32_t vw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) vw[e] = 0u;
    if (present != 0u)
        make_group<T, D, VEC, false>(at, g, present, [&](int r) { return k + (src + r) * D; }, [&](int r) { return v + (src + r) * D; }, vw);
    if (E == 4) *reinterpret_cast<uint4*>(&s_words[g][lane * E]) = make_uint4(vw[0], vw[1], vw[E - 2], vw[E - 1]);
    else *reinterpret_cast<uint2*>(&s_words[g][lane * E]) = make_uint2(vw[0], vw[1]);
    __syncthreads();
    if (tid < D) {
        const uint32_t o[4] = {old.x, old.y, old.z, old.w};
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = s_words[j][tid] | (o[j] & ~nibbles_of((rows >> (j * kGroup)) & 0xFFu));
        *dst = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// One warp per (layer, sequence, head): the rows it commits lie in one group or a few.
template <typename T, int D>
__global__ void __launch_bounds__(kStoreThreads)
commit_kv4_kernel(void* const* __restrict__ cache_layers, const void* const* __restrict__ k_tree_layers,
                  const void* const* __restrict__ v_tree_layers, const int32_t* __restrict__ seq_lens,
                  const int32_t* __restrict__ accept_len, const int32_t* __restrict__ out_nodes,
                  const int32_t* __restrict__ best_root, int n_levels, int BH, int H, int N, int pages) {
    constexpr int E = D / 32;
    const int bh = blockIdx.x * kStoreWarps + (threadIdx.x >> 5), b = bh / H, layer = blockIdx.y, lane = threadIdx.x & 31;
    if (bh >= BH) return;
    const int L_max = pages * kPageRows;
    const int L = min(max(seq_lens[b], 0), L_max);
    const int acc = min(max(accept_len[b], 0), n_levels);
    const int end = min(L + 1 + acc, L_max);                  // rows beyond the cache are dropped
    const T* const kt = static_cast<const T*>(k_tree_layers[layer]) + (size_t)bh * N * D;
    const T* const vt = static_cast<const T*>(v_tree_layers[layer]) + (size_t)bh * N * D;
    unsigned char* const head = static_cast<unsigned char*>(cache_layers[layer]) + (size_t)bh * pages * kv4_page_bytes(D);
    // (the pointers come from a table on the device, so their alignment is only known here)
    const bool vec = ((reinterpret_cast<uintptr_t>(kt) | reinterpret_cast<uintptr_t>(vt)) & 15u) == 0;
    for (int row0 = L / kGroup * kGroup; row0 < end; row0 += kGroup) {
        unsigned char* const at = head + (size_t)(row0 / kPageRows) * kv4_page_bytes(D);
        const int g = row0 % kPageRows / kGroup;
        // lane r: the tree node of row row0 + r (the winning root first, then the accepted nodes)
        int node = -1;
        const int row = row0 + lane;
        if (lane < kGroup && row >= L && row < end) node = row == L ? best_root[b] : out_nodes[(size_t)b * n_levels + (row - L - 1)];
        if (node >= N) node = -1;                             // malformed verify output: leave the row alone
        const uint32_t present = __ballot_sync(0xffffffffu, node >= 0);
        if (present == 0u) continue;
        uint32_t old[E], vw[E];
        uint32_t* const dst = reinterpret_cast<uint32_t*>(at + kv4_values_at(D) + lane * E * 16 + g * 4);
#pragma unroll
        for (int e = 0; e < E; ++e) old[e] = present == 0xFFu ? 0u : dst[e * 4];
        auto k_row = [&](int r) { return kt + (size_t)__shfl_sync(0xffffffffu, node, r) * D; };
        auto v_row = [&](int r) { return vt + (size_t)__shfl_sync(0xffffffffu, node, r) * D; };
        if (vec) make_group<T, D, true, true>(at, g, present, k_row, v_row, vw);
        else make_group<T, D, false, true>(at, g, present, k_row, v_row, vw);
        const uint32_t keep = ~nibbles_of(present);
#pragma unroll
        for (int e = 0; e < E; ++e) dst[e * 4] = vw[e] | (old[e] & keep);
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
    __shared__ alignas(16) unsigned char s_codes[kPageRows][D];   // value codes by row, one byte each
    const int bh = blockIdx.y, b = bh / H, layer = blockIdx.z, tid = threadIdx.x;
    const long long first = first_rows[b];
    const int n = n_rows ? min(max(n_rows[b], 0), T_rows) : T_rows;
    const long long page = (first >= 0 ? first / kPageRows : -((-first + kPageRows - 1) / kPageRows)) + blockIdx.x;
    const long long row0 = page * kPageRows;                  // the page's rows are rows row0 - first .. of k and v
    const int r0 = (int)max(first - row0, 0LL), r1 = (int)min(first + T_rows - row0, (long long)kPageRows);
    if (r0 >= r1) return;
    const bool there = page >= 0 && page < pages;
    const unsigned char* at = static_cast<const unsigned char*>(cache_layers[layer]) + ((size_t)bh * pages + (there ? page : 0)) * kv4_page_bytes(D);
    const unsigned short* const sc = reinterpret_cast<const unsigned short*>(at + kv4_scales_at(D));
    const size_t out0 = ((size_t)layer * gridDim.y + bh) * T_rows;
    // all that the block reads is on its way before the first of it is used
    constexpr int U = kPageRows * (D / 8) / kStoreThreads;    // pieces of eight channels per thread
    const int pieces = (r1 - r0) * (D / 8);
    uint4 vals = make_uint4(0, 0, 0, 0);
    if (there && tid < D) vals = *reinterpret_cast<const uint4*>(at + kv4_values_at(D) + tid * 16);
    uint32_t keys[U], k_scale[U], v_scale[U];                 // scale in the low half, offset in the high half
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = tid + u * kStoreThreads, r = r0 + i / (D / 8), c = i % (D / 8);
        keys[u] = k_scale[u] = v_scale[u] = 0u;               // rows that are not there read as zero
        if (there && i < pieces && (int)(row0 + r - first) < n) {
            keys[u] = *reinterpret_cast<const uint32_t*>(at + (c >> 2) * (kPageRows * 16) + r * 16 + (c & 3) * 4);
            k_scale[u] = sc[r] | ((uint32_t)sc[kPageRows + r] << 16);
            v_scale[u] = sc[2 * kPageRows + r] | ((uint32_t)sc[3 * kPageRows + r] << 16);
        }
    }
    if (tid < D) {
        const uint32_t w[4] = {vals.x, vals.y, vals.z, vals.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (8 * j + 8 <= r0 || 8 * j >= r1) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) s_codes[8 * j + e][tid] = (unsigned char)((w[j] >> kv4_bit(e)) & 15u);
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = tid + u * kStoreThreads, r = r0 + i / (D / 8), c = i % (D / 8);
        if (i >= pieces) break;
        const int t = (int)(row0 + r - first);
        const uint2 codes = *reinterpret_cast<const uint2*>(&s_codes[r][8 * c]);
        const float ks = bf16_bits_to_f32(k_scale[u] & 0xFFFFu), ko = __uint_as_float(k_scale[u] & 0xFFFF0000u);
        const float vs = bf16_bits_to_f32(v_scale[u] & 0xFFFFu), vo = __uint_as_float(v_scale[u] & 0xFFFF0000u);
        float xk[8], xv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            xk[e] = kv4_value((keys[u] >> kv4_bit(e)) & 15u, ks, ko);
            xv[e] = kv4_value(((e < 4 ? codes.x : codes.y) >> (8 * (e & 3))) & 15u, vs, vo);
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
        commit_kv4_kernel<T_, D_><<<dim3((unsigned)((B * H + kStoreWarps - 1) / kStoreWarps), (unsigned)n_layers), kStoreThreads, 0, s>>>(
            cache_layers, k_tree_layers, v_tree_layers, seq_lens, accept_len, out_nodes, best_root, n_levels, B * H, H, N, L_max / kPageRows);
        MCSD_CUDA_CHECK(cudaGetLastError());
        grow_lens_kernel<<<(B + 127) / 128, 128, 0, s>>>(seq_lens, accept_len, n_levels, B, L_max);
        MCSD_CUDA_CHECK(cudaGetLastError());
        count_launches(2);
        return MCSD_OK;
    });
}
