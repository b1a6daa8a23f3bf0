// Candidates from next-token logits: temperature, top-k, top-p and min-p, the probabilities that are left, and inverse-CDF
// draws from caller-supplied uniforms (the draft's side of Fig. 1 step 1, and the rows p and q of its verification).
//
//   w_i = exp((l_i - max) / T);  every filter keeps a prefix of the tokens in the order (larger logit, then lower id):
//   top-k the first k, top-p the shortest prefix of those whose mass reaches top_p of theirs, min-p those with w_i >= min_p.
//   So what is kept is a cut (logit, id), and p_i = w_i / (sum of w over what is before the cut).
//
// Weights are summed as whole numbers of 2^-31, so that a sum does not depend on its order: filters, draws and
// probabilities are the same whatever the number of blocks, and from run to run.  A rounding to 2^-31 is half a step, and the
// largest weight is 1: a sum over V tokens is off by at most V 2^-32 of it (3e-5 for 131072 tokens whose weights all round
// alike, 2e-8 where they do not).
//
// A row is read once and lies in shared memory from then on, split by columns over a cluster of blocks: one block as long as
// it fits, more where there are fewer rows than multiprocessors.  A cut is found from a histogram over 1024 steps of
// (max - l), linear over the part that carries mass; the tokens of the step where the sum crosses (some hundred) are
// collected and placed by counting, every one against every other.  Steps that hold more tokens than that (equal logits,
// masked ones, steep rows) are split again, in the order of (logit, id), 1024 ways a pass.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace mcsd {

constexpr int kSampleThreads = 1024, kSampleWarps = kSampleThreads / 32;
constexpr int kSampleMaxSegment = 32768;      // tokens of a block
constexpr int kSampleMaxVocab = 8 * kSampleMaxSegment;
constexpr int kChunk = 128;                   // tokens of a partial sum
constexpr int kBins = 1024;
constexpr int kListMax = 1024;                // tokens that are placed by counting
constexpr float kBinSpan = 20.0f;             // the first histogram reaches down to exp(-20) of the largest weight

typedef unsigned long long u64;

struct SampleArgs {
    const void* logits;
    long long row_stride;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* tokens;
    float* probs;
    int V, K, segment;
    bool vec_in, vec_out;
};

struct alignas(16) SampleShared {
    uint32_t lo[kBins], hi[kBins];            // sums of a step, low and high words
    u64 scan[kSampleWarps];
    u64 chunk[kSampleMaxSegment / kChunk + 1];
    float red[kSampleWarps];
    u64 total;                                // this block's kept mass
    float block_max;
    // decision of a pass
    int bin;
    u64 before;                               // mass or count before that step
    u64 range_lo, range_hi;                   // smallest and largest place among the step's tokens (this block's part)
    int list_n;                               // tokens collected (first block of the cluster)
    u64 cut;                                  // place of the last token kept
    u64 cut_sum;                              // sum up to and with it
    u64 list_place[kListMax];
    uint32_t list_f[kListMax];
};
static_assert(sizeof(SampleShared) % 16 == 0, "the logits behind it are read as 16-byte vectors");

// a token's place: smaller is earlier in the order (larger logit, lower id)
__device__ __forceinline__ u64 place_of(float l, uint32_t id) {
    const uint32_t x = __float_as_uint(l == 0.0f ? 0.0f : l);               // -0 and 0 are equal
    const uint32_t up = (x & 0x80000000u) ? ~x : x | 0x80000000u;           // grows with l
    return ((u64)(~up) << 32) | id;
}

struct Row {
    const float* data;        // this block's logits
    int n, first;             // how many, id of the first
    float top;                // largest logit of the row
    float c_hi, c_lo;         // log2(e) / T
    float bin_scale;
};

__device__ __forceinline__ float below_top(const Row& r, float l) { return l == r.top ? 0.0f : r.top - l; }
// exp((l - top) / T) to about two units in the last place: the exponent's rounding is carried along
__device__ __forceinline__ float weight(const Row& r, float l) {
    const float d = below_top(r, l), e = d * r.c_hi;
    if (!(e < 140.0f)) return 0.0f;
    const float rest = fmaf(d, r.c_hi, -e) + d * r.c_lo;
    const float w = exp2f(-e);
    return fmaf(-rest * 0.69314718f, w, w);
}
// w (0 .. 1) in steps of 2^-31, nearest: by adding a number whose last place is 1, twice, no conversion instruction
__device__ __forceinline__ uint32_t fixed31(float w) {
    const float big = 12582912.0f;                                            // 1.5 * 2^23
    const float a = w * 1048576.0f, t = a + big, rest = a - (t - big);
    const float t2 = fmaf(rest, 2048.0f, big);
    return (uint32_t)(__float_as_int(t) - 0x4B400000) * 2048u + (uint32_t)(__float_as_int(t2) - 0x4B400000);
}
__device__ __forceinline__ int bin_of(const Row& r, float l) {
    const float x = fminf(below_top(r, l) * r.bin_scale, (float)(kBins - 1));  // NaN cannot occur: top is finite or l == top
    return (int)x;
}

__device__ __forceinline__ u64 warp_scan(u64 v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

template <bool MASS>
__device__ __forceinline__ void hist_add(SampleShared* sh, int bin, uint32_t f) {
    if (MASS) {
        if (f == 0) return;
        const uint32_t old = atomicAdd(&sh->lo[bin], f);
        if (old + f < old) atomicAdd(&sh->hi[bin], 1u);
    } else {
        atomicAdd(&sh->lo[bin], 1u);
    }
}

__device__ __forceinline__ void clear_hist(SampleShared* sh) {
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { sh->lo[i] = 0; sh->hi[i] = 0; }
}

// The step in which the sum over steps passes `target`, over all blocks' histograms; every block finds the same.
// Written to sh->bin and sh->before (sh->before starts as the sum before the first step).
__device__ void find_bin(SampleShared* sh, cg::cluster_group& cluster, int ranks, u64 start, u64 target) {
    cluster.sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    u64 v = 0;
    for (int r = 0; r < ranks; ++r) {
        const SampleShared* o = ranks == 1 ? sh : cluster.map_shared_rank(sh, r);
        v += ((u64)o->hi[tid] << 32) + o->lo[tid];
    }
    if (tid == 0) sh->bin = kBins;                                            // no step: the target is beyond the sum
    u64 in = warp_scan(v, lane);
    if (lane == 31) sh->scan[warp] = in;
    __syncthreads();
    for (int w = 0; w < warp; ++w) in += sh->scan[w];
    in += start;
    if (in - v < target && target <= in) { sh->bin = tid; sh->before = in - v; }
    cluster.sync();                                                           // histograms have been read, decision is there
}

// The cut: the token at which the sum of f (MASS) or the count over the order passes `target` (1 .. sum).  `limit` is a cut
// found before: tokens behind it do not take part.
template <bool MASS>
__device__ void select_cut(SampleShared* sh, cg::cluster_group& cluster, int ranks, const Row& r, u64 target, u64 limit) {
    const int tid = threadIdx.x;
    clear_hist(sh);
    if (tid == 0) { sh->list_n = 0; sh->range_lo = ~0ull; sh->range_hi = 0; }
    __syncthreads();
    for (int i = tid; i < r.n; i += kSampleThreads) {
        const float l = r.data[i];
        if (l == -INFINITY || place_of(l, r.first + i) > limit) continue;
        hist_add<MASS>(sh, bin_of(r, l), MASS ? fixed31(weight(r, l)) : 0u);
    }
    find_bin(sh, cluster, ranks, 0, target);
    const int bin = sh->bin;
    u64 before = sh->before, lo = 0, hi = ~0ull;
    SampleShared* first = ranks == 1 ? sh : cluster.map_shared_rank(sh, 0);
    for (;;) {
        // collect the tokens of the step [lo, hi]; the first block holds the list
        u64 mn = ~0ull, mx = 0;
        for (int i = tid; i < r.n; i += kSampleThreads) {
            const float l = r.data[i];
            if (l == -INFINITY || bin_of(r, l) != bin) continue;
            const u64 p = place_of(l, r.first + i);
            if (p > limit || p < lo || p > hi) continue;
            mn = min(mn, p);
            mx = max(mx, p);
            const int at = atomicAdd(&first->list_n, 1);
            if (at < kListMax) {
                first->list_place[at] = p;
                first->list_f[at] = MASS ? fixed31(weight(r, l)) : 1u;
            }
        }
        if (mn != ~0ull) { atomicMin(&sh->range_lo, mn); atomicMax(&sh->range_hi, mx); }
        cluster.sync();
        const int n = first->list_n;
        if (n <= kListMax) {
            // place by counting, in the first block: a few threads a token, each a part of the list
            if (ranks == 1 || cluster.block_rank() == 0) {
                const int per = max(1, min(32, kSampleThreads / max(n, 1)));
                int width = 1;
                while (width * 2 <= per) width *= 2;                          // threads a token: a power of two, inside a warp
                for (int i0 = 0; i0 < n; i0 += kSampleThreads / width) {
                    const int i = i0 + tid / width, part = tid % width;
                    u64 sum = 0;
                    const u64 p = i < n ? sh->list_place[i] : 0;
                    if (i < n)
                        for (int j = part; j < n; j += width)
                            if (sh->list_place[j] < p) sum += sh->list_f[j];
                    for (int o = width / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if (i < n && part == 0) {
                        const u64 b = before + sum;
                        if (b < target && target <= b + sh->list_f[i]) { sh->cut = p; sh->cut_sum = b + sh->list_f[i]; }
                    }
                }
            }
            cluster.sync();
            if (ranks > 1 && cluster.block_rank() != 0 && tid == 0) { sh->cut = first->cut; sh->cut_sum = first->cut_sum; }
            cluster.sync();
            return;
        }
        // too many: split the range of places
        u64 a = ~0ull, z = 0;
        for (int k = 0; k < ranks; ++k) {
            const SampleShared* o = ranks == 1 ? sh : cluster.map_shared_rank(sh, k);
            a = min(a, o->range_lo);
            z = max(z, o->range_hi);
        }
        cluster.sync();
        int shift = 0;
        while (((z - a) >> shift) >= (u64)kBins) ++shift;
        clear_hist(sh);
        if (tid == 0) { sh->list_n = 0; sh->range_lo = ~0ull; sh->range_hi = 0; }
        __syncthreads();
        for (int i = tid; i < r.n; i += kSampleThreads) {
            const float l = r.data[i];
            if (l == -INFINITY || bin_of(r, l) != bin) continue;
            const u64 p = place_of(l, r.first + i);
            if (p > limit || p < a || p > z) continue;
            hist_add<MASS>(sh, (int)((p - a) >> shift), MASS ? fixed31(weight(r, l)) : 0u);
        }
        find_bin(sh, cluster, ranks, before, target);
        before = sh->before;
        lo = a + ((u64)sh->bin << shift);
        hi = min(z, lo + (((u64)1 << shift) - 1));
        __syncthreads();
    }
}

// sum of f over the cluster's tokens up to `limit`
__device__ u64 mass_up_to(SampleShared* sh, cg::cluster_group& cluster, int ranks, const Row& r, u64 limit) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    u64 sum = 0;
    for (int i = tid; i < r.n; i += kSampleThreads) {
        const float l = r.data[i];
        if (l != -INFINITY && place_of(l, r.first + i) <= limit) sum += fixed31(weight(r, l));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sh->scan[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        u64 v = sh->scan[lane];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) sh->total = v;
    }
    cluster.sync();
    u64 all = 0;
    for (int k = 0; k < ranks; ++k) all += (ranks == 1 ? sh : cluster.map_shared_rank(sh, k))->total;
    cluster.sync();
    return all;
}

template <typename T> __device__ __forceinline__ float logit_of(T x);
template <> __device__ __forceinline__ float logit_of(float x) { return x; }
template <> __device__ __forceinline__ float logit_of(__nv_bfloat16 x) { return __bfloat162float(x); }

// grid: rows * cluster size
template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 1) sample_kernel(const __grid_constant__ SampleArgs a) {
    extern __shared__ float4 raw4[];
    SampleShared* sh = reinterpret_cast<SampleShared*>(raw4);
    float* data = reinterpret_cast<float*>(sh + 1);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const long long row = blockIdx.x / ranks;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int first = rank * a.segment, n = max(0, min(a.segment, a.V - first));
    const T* src = static_cast<const T*>(a.logits) + row * a.row_stride + first;

    // ---- the row into shared memory, NaN as -infinity, and its largest logit
    float mx = -INFINITY;
    constexpr int kVec = 16 / sizeof(T);
    int done = 0;
    if (a.vec_in) {
        done = n / kVec * kVec;
#pragma unroll 4
        for (int i = tid * kVec; i < done; i += kSampleThreads * kVec) {
            alignas(16) T t[kVec];
            *reinterpret_cast<uint4*>(t) = __ldcs(reinterpret_cast<const uint4*>(src + i));
            float v[kVec];
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                v[j] = logit_of<T>(t[j]);
                if (isnan(v[j])) v[j] = -INFINITY;
                mx = fmaxf(mx, v[j]);
            }
#pragma unroll
            for (int j = 0; j < kVec; j += 4) *reinterpret_cast<float4*>(data + i + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
    }
#pragma unroll 8
    for (int i = done + tid; i < n; i += kSampleThreads) {
        float v = logit_of<T>(src[i]);
        if (isnan(v)) v = -INFINITY;
        mx = fmaxf(mx, v);
        data[i] = v;
    }
    const int padded = (n + kChunk - 1) / kChunk * kChunk;
    for (int i = n + tid; i < padded; i += kSampleThreads) data[i] = -INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) sh->red[warp] = mx;
    __syncthreads();
    if (warp == 0) {
        float v = sh->red[lane];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        if (lane == 0) sh->block_max = v;
    }
    cluster.sync();
    float top = -INFINITY;
    for (int k = 0; k < ranks; ++k) top = fmaxf(top, (ranks == 1 ? sh : cluster.map_shared_rank(sh, k))->block_max);

    // ---- the filters of this row
    const float T_in = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = !(T_in > 0.0f);
    const double inv = 1.4426950408889634 / (greedy ? 1.0 : (double)T_in);
    Row r;
    r.data = data; r.n = n; r.first = first; r.top = top;
    r.c_hi = (float)fmin(inv, 1e38);                     // a temperature near zero: finite, so that the top keeps weight 1
    r.c_lo = inv < 1e38 ? (float)(inv - (double)r.c_hi) : 0.0f;
    r.bin_scale = fminf((float)((double)kBins / (kBinSpan * (greedy ? 1.0 : (double)T_in))), 1e30f);
    int k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
    const float tp = greedy || !a.top_p ? 1.0f : a.top_p[row], mp = greedy || !a.min_p ? 0.0f : a.min_p[row];
    u64 cut = ~0ull;
    if (top > -INFINITY) {
        if (k > 0 && k < a.V) {
            // fewer than k tokens may be left of a masked row: find_bin then reports no step
            clear_hist(sh);
            __syncthreads();
            int mine = 0;
            for (int i = tid; i < n; i += kSampleThreads) mine += data[i] != -INFINITY;
            mine = __reduce_add_sync(0xffffffffu, mine);
            if (lane == 0) atomicAdd(&sh->lo[0], (uint32_t)mine);
            cluster.sync();
            u64 live = 0;
            for (int q = 0; q < ranks; ++q) live += (ranks == 1 ? sh : cluster.map_shared_rank(sh, q))->lo[0];
            cluster.sync();
            if ((u64)k < live) {
                select_cut<false>(sh, cluster, ranks, r, (u64)k, ~0ull);
                cut = sh->cut;
            }
        }
        if (tp < 1.0f) {
            const u64 total = mass_up_to(sh, cluster, ranks, r, cut);
            const double want = ceil((double)total * (double)fmaxf(tp, 0.0f));
            const u64 target = min(total, max((u64)1, (u64)want));
            select_cut<true>(sh, cluster, ranks, r, target, cut);
            cut = sh->cut;
        }
    }

    // ---- weights of what is kept, their sums by chunks of 128
    __syncthreads();
    const float floor_w = mp > 0.0f ? fminf(mp, 1.0f) : 0.0f;
    const int chunks = padded / kChunk;
    for (int c = warp; c < chunks; c += kSampleWarps) {
        float4 v = *reinterpret_cast<const float4*>(data + c * kChunk + lane * 4);
        float* e = reinterpret_cast<float*>(&v);
        uint32_t hi = 0, lo = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float l = e[j];
            float w = 0.0f;
            if (l != -INFINITY && place_of(l, first + c * kChunk + lane * 4 + j) <= cut) {
                w = weight(r, l);
                if (w < floor_w) w = 0.0f;
            }
            e[j] = w;
            const uint32_t f = fixed31(w);
            hi += f >> 16;
            lo += f & 0xffffu;
        }
        *reinterpret_cast<float4*>(data + c * kChunk + lane * 4) = v;
        hi = __reduce_add_sync(0xffffffffu, hi);
        lo = __reduce_add_sync(0xffffffffu, lo);
        if (lane == 0) sh->chunk[c + 1] = ((u64)hi << 16) + lo;
    }
    __syncthreads();
    if (warp == 0) {                                     // running sums of at most 256 chunks
        u64 base = 0;
        if (lane == 0) sh->chunk[0] = 0;
        for (int c0 = 0; c0 < chunks; c0 += 32) {
            const u64 v = c0 + lane < chunks ? sh->chunk[c0 + lane + 1] : 0;
            const u64 s = base + warp_scan(v, lane);
            if (c0 + lane < chunks) sh->chunk[c0 + lane + 1] = s;
            base = __shfl_sync(0xffffffffu, s, 31);
        }
        if (lane == 0) sh->total = base;
    }
    cluster.sync();
    u64 all = 0, mine0 = 0;
    for (int q = 0; q < ranks; ++q) {
        const u64 t = (ranks == 1 ? sh : cluster.map_shared_rank(sh, q))->total;
        if (q < rank) mine0 += t;
        all += t;
    }
    const u64 mine1 = mine0 + sh->total;

    // ---- draws: the first token at which the running sum passes u * sum
    if (a.tokens) {
        for (int j = warp; j < a.K; j += kSampleWarps) {
            int32_t* out = a.tokens + row * a.K + j;
            if (all == 0) {                              // no token left: every logit is -infinity or NaN
                if (rank == 0 && lane == 0) *out = -1;
                continue;
            }
            const double x = (double)a.u[row * a.K + j] * (double)all;
            const u64 t = x > 0.0 ? min(all - 1, (u64)x) : 0;
            if (t < mine0 || t >= mine1) continue;       // another block's
            const u64 at = t - mine0;
            int lo = 0, hi = chunks;                     // chunk[lo] <= at < chunk[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sh->chunk[mid] <= at) lo = mid; else hi = mid;
            }
            const float4 v = *reinterpret_cast<const float4*>(data + lo * kChunk + lane * 4);
            const float e[4] = {v.x, v.y, v.z, v.w};
            u64 own = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) own += fixed31(e[i]);
            const u64 end = sh->chunk[lo] + warp_scan(own, lane);
            u64 s = end - own;
            if (s <= at && at < end) {
                int id = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u64 f = fixed31(e[i]);
                    if (s <= at && at < s + f) id = first + lo * kChunk + lane * 4 + i;
                    s += f;
                }
                *out = id;
            }
        }
    }
    // ---- probabilities
    if (a.probs) {
        const float scale = all ? (float)(2147483648.0 / (double)all) : 0.0f;
        float* dst = a.probs + row * a.V + first;
        if (a.vec_out) {
            for (int i = tid * 4; i < n; i += kSampleThreads * 4) {
                float4 v = *reinterpret_cast<const float4*>(data + i);
                v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
                __stcs(reinterpret_cast<float4*>(dst + i), v);
            }
        } else {
            for (int i = tid; i < n; i += kSampleThreads) __stcs(dst + i, data[i] * scale);
        }
    }
    cluster.sync();                                      // no block leaves while another may read its shared memory
}

}  // namespace mcsd

extern "C" int mcsd_sample_candidates(const void* logits, long long row_stride, int dtype, int rows, int V, const float* temperature,
                                      const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int K,
                                      int32_t* tokens, float* probs, void* stream) {
    if (!logits || (!tokens && !probs) || (tokens && !u)) return MCSD_ERR_NULL;
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (rows < 1 || rows > (1 << 24) || V < 1 || V > mcsd::kSampleMaxVocab || row_stride < V || K < 0 || (tokens && K < 1) || K > 1024)
        return MCSD_ERR_BAD_SHAPE;
    int dev = 0, sms = 0;
    MCSD_CUDA_CHECK(cudaGetDevice(&dev));
    MCSD_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // blocks a row: enough for the row to fit, then more while there are multiprocessors without a row
    int c = 1;
    while ((long long)c * mcsd::kSampleMaxSegment < V) c *= 2;
    while (c < 8 && (long long)rows * c * 2 <= sms && V / (c * 2) >= 1024) c *= 2;
    mcsd::SampleArgs a{};
    a.logits = logits; a.row_stride = row_stride;
    a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u;
    a.tokens = tokens; a.probs = probs;
    a.V = V; a.K = K;
    a.segment = ((V + c - 1) / c + mcsd::kChunk - 1) / mcsd::kChunk * mcsd::kChunk;
    const int elt = dtype == MCSD_F32 ? 4 : 2;
    a.vec_in = (reinterpret_cast<uintptr_t>(logits) & 15u) == 0 && (row_stride * elt) % 16 == 0;
    a.vec_out = probs && (reinterpret_cast<uintptr_t>(probs) & 15u) == 0 && V % 4 == 0;
    const int smem = (int)sizeof(mcsd::SampleShared) + a.segment * (int)sizeof(float);
    auto kernel = dtype == MCSD_F32 ? mcsd::sample_kernel<float> : mcsd::sample_kernel<__nv_bfloat16>;
    MCSD_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)rows * c);
    cfg.blockDim = dim3(mcsd::kSampleThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = c; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, a));
    mcsd::count_launches(1);
    return MCSD_OK;
}
