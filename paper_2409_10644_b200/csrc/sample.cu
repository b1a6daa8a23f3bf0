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
// alike, 2e-8 where they do not).  A kept token of half a step or less, 2^-32 of the largest, counts as nothing in a sum: it has
// its probability and is never drawn.  All such tokens of a row together have at most V 2^-32 (6e-5 for 262144).
//
// A row is read from memory once; what looks at it again finds it in L2, so that shared memory holds only what was found, and two
// blocks share a multiprocessor: one row's chain of short steps runs under the other's.  (With the row in shared memory and one
// block a multiprocessor 720 rows of 32000 took 103 us, with a row over two blocks 114; with three blocks of 40 registers 139.)  A block takes a row; where there are fewer
// rows than multiprocessors a cluster of up to eight takes it, split by columns (a meeting of a cluster costs a microsecond, ten
// times one of a block).  The first pass finds the largest logit; the second, a comparison a token, picks the few that can decide
// anything, and all later work is on those:
//   * top-k: the k-th largest of the threads' own maxima (of those of four tokens, for a large k: 2000 of 32000, 720 rows 132 us,
//     350 without) bounds the k-th largest logit from below; the tokens down to that bound are hardly more than k;
//   * top-p alone: the tokens from 2^-14 of the largest on; the weights of the others are only added up.  (Where the cut turns
//     out to be among those, the pass is made again for all tokens.)  Where they are more than the list holds, a pass adds up
//     what lies below 2^-10 .. 2^-13, and a higher bound is taken if that allows it;
//   * once the cut is known, a list that overflowed is made again of what is kept (at temperature 1 and top_p 0.95 of normal
//     logits three units wide, 720 rows of 32000: 180 us; 278 with passes over the row from there on; 329 at temperature 1.3,
//     where no bound is high enough and the cut is found by passes over the row).
// Tokens that may hold the cut are collected in the cluster's first block: all of them under top-k, under top-p alone those of the
// step of a histogram (1024 steps of (max - l), linear over the part that carries mass) in which the sum crosses.  On that list
// the cut is found by dividing its range of places 1024 ways until 32 tokens are left, which a warp compares.  A list that
// overflows (equal logits, masked ones, a large k) is divided in the same way by passes over the row.
// What bounds it: latency.  720 rows of 32000 take 90 us (184 MB in and out, 2.0 TB/s; 39 % of the issue slots, the two blocks of a
// multiprocessor waiting half of their time for memory or for one another), one row 17 us, 16 rows of 131071 32 us (of which
// six meetings, two readings and the cut).
// Probabilities are zeros and a value for each token that is kept.  They are written last, behind all meetings of the cluster
// but one that orders nothing: a meeting waits for the writes before it (1 us each).
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cstddef>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace mcsd {

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kSampleMaxVocab = 262144;
constexpr int kChunk = 128;                   // tokens of a partial sum
constexpr int kBins = 2 * kSampleThreads;
constexpr int kListMax = 3000;                // tokens of the first block's list
constexpr int kPickMax = 6144;                // tokens that a block lists as picked (what two blocks leave of 196 KB); with more it
                                              // goes through the row each time
constexpr int kListK = 2560;                  // top-k that is tried on a list
constexpr float kBinSpan = 20.0f;             // the first histogram reaches down to exp(-20) of the largest weight
constexpr int kSteps = 4;                     // thresholds between there and 2^-10
constexpr float kTail = 14.0f;                // tokens below 2^-14 of the largest are added up without a step of their own

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
    u64 list[kListMax];                       // places
    u64 few[32];
    alignas(16) uint32_t lo[kBins], hi[kBins];   // sums of a step, low and high words
    int few_n;
    u64 scan[kSampleWarps];
    u64 chunk[kSampleMaxVocab / kChunk + 1];
    float red[kSampleWarps];
    int red_live[kSampleWarps];
    float block_max;
    int block_live;                           // tokens that are not -infinity
    u64 total;                                // this block's kept mass
    u64 tail;                                 // mass below the steps
    int bin;                                  // the step that was found, or kBins
    u64 before;                               // mass or count before that step
    u64 target;
    float c_hi, c_lo, bin_scale, scale;       // of the row, worked out by one thread: 64-bit arithmetic by all takes microseconds
    u64 range_lo, range_hi;                   // smallest and largest place among the step's tokens (this block's part)
    int list_n;                               // tokens collected (first block of the cluster)
    u64 cut;                                  // place of the last token kept
    int picked;                               // tokens picked (more than kPickMax: none are listed)
    u64 below[kSteps + 1];                    // weight of all, and of what lies below some thresholds, in steps of 2^-20
    int pick[kPickMax];
    float pick_l[kPickMax];                   // their logits, later their weights
};
static_assert(offsetof(SampleShared, lo) % 8 == 0 && offsetof(SampleShared, hi) % 8 == 0, "steps are read in pairs");
static_assert(2 * (sizeof(SampleShared) + 1024) <= 228 * 1024, "two blocks a multiprocessor");

// a token's place: smaller is earlier in the order (larger logit, lower id)
__device__ __forceinline__ u64 place_of(float l, uint32_t id) {
    const uint32_t x = __float_as_uint(l == 0.0f ? 0.0f : l);               // -0 and 0 are equal
    const uint32_t up = (x & 0x80000000u) ? ~x : x | 0x80000000u;           // grows with l
    return ((u64)(~up) << 32) | id;
}

template <typename T> __device__ __forceinline__ float logit_of(T x);
template <> __device__ __forceinline__ float logit_of(float x) { return x; }
template <> __device__ __forceinline__ float logit_of(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float no_nan(float x) { return isnan(x) ? -INFINITY : x; }

struct Scale {
    float top;                // largest logit of the row
    float c_hi, c_lo;         // log2(e) / T
    float bin_scale;
};
template <typename T>
struct Row : Scale {
    const T* data;            // this block's logits
    int n, first, whole;      // how many, id of the first, tokens of all blocks
    bool vec;                 // four at a time
    __device__ __forceinline__ float at(int i) const { return no_nan(logit_of<T>(data[i])); }
    // tokens i .. i + 3, -infinity past the end; i a multiple of four
    __device__ __forceinline__ float4 four(int i) const {
        float4 v;
        if (vec && i + 4 <= n) {
            if constexpr (sizeof(T) == 4) {
                v = *reinterpret_cast<const float4*>(data + i);
            } else {
                const uint2 w = *reinterpret_cast<const uint2*>(data + i);
                v = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
            }
            return make_float4(no_nan(v.x), no_nan(v.y), no_nan(v.z), no_nan(v.w));
        }
        if (i >= n) return make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        v.x = i < n ? at(i) : -INFINITY;
        v.y = i + 1 < n ? at(i + 1) : -INFINITY;
        v.z = i + 2 < n ? at(i + 2) : -INFINITY;
        v.w = i + 3 < n ? at(i + 3) : -INFINITY;
        return v;
    }
};

__device__ __forceinline__ float below_top(const Scale& r, float l) { return l == r.top ? 0.0f : r.top - l; }
// exp((l - top) / T).  The difference is rounded to 32 bits, which moves a weight by 2^-24 ln(1 / w) of itself (1.3e-6 at 2^-31, less
// the heavier it is); behind it the exponent's rounding is carried along, so that about two units in the last place come on top.
__device__ __forceinline__ float weight(const Scale& r, float l) {
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
// The weight as filters add it up.  Small ones are added by the hundred of thousands while the row is read: an approximate
// exponential, in steps of 2^-31 by adding it to 1.5 * 2^23 (below 2^21.5 they stand in the last places).  Its exponent is
// rounded three times (the difference, log2(e) / T and their product, 2^-24 each), which makes 3 * 2^-24 * ln 2 * 32 = 4e-6 where
// the weight is 2^-32 and 1.2e-6 where it is 2^-9.5, and the instruction adds 2^-22.  Wherever a token is met its weight is the same.
constexpr float kSmall = 9.5f;
__device__ __forceinline__ uint32_t small31(float e) {                        // 2^e
    float w;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(e));
    return (uint32_t)__float_as_int(fmaf(w, 2147483648.0f, 12582912.0f)) - 0x4B400000u;
}
__device__ __forceinline__ uint32_t mass31(const Scale& r, float l) {
    const float e = (l - r.top) * r.c_hi;
    return e < -kSmall ? small31(e) : fixed31(weight(r, l));
}
__device__ __forceinline__ int bin_of(const Scale& r, float l) {
    const float x = fminf(below_top(r, l) * r.bin_scale, (float)(kBins - 1));  // NaN cannot occur: top is finite or l == top
    return (int)x;
}

// a logit that lies below all of a step's, by little
__device__ __forceinline__ float step_floor(const Scale& r, int bin) {
    if (bin >= kBins - 1) return -INFINITY;
    const float d = (float)(bin + 1) / r.bin_scale;
    const float l = r.top - d * 1.00001f;
    return l - fabsf(l) * 1e-6f > -INFINITY ? l - fabsf(l) * 1e-6f : -INFINITY;    // also where it is no number
}
__device__ __forceinline__ float logit_at(u64 place) {                        // the inverse of place_of
    const uint32_t up = ~(uint32_t)(place >> 32);
    return __uint_as_float((up & 0x80000000u) ? up ^ 0x80000000u : ~up);
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

// Picks the tokens whose logit is at least `least`; with TAILS, returns this thread's sum of the others' weights, which are
// below 2^-10 at most (in steps of 2^-31 below 2^21: added to 1.5 * 2^23 a weight stands in the last places).
template <bool TAILS, typename T>
__device__ __forceinline__ u64 pick_tokens(SampleShared* sh, const Row<T>& r, float least) {
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) sh->picked = 0;
    __syncthreads();
    u64 tail = 0;
    for (int base0 = 4 * tid; base0 < r.n; base0 += 32 * kSampleThreads) {        // a bit a token, 32 tokens of a thread at a time
        uint32_t picks = 0;
        float4 v4[8];
#pragma unroll
        for (int it = 0; it < 8; ++it) v4[it] = r.four(base0 + it * 4 * kSampleThreads);
#pragma unroll
        for (int it = 0; it < 8; ++it) {
            const float v[4] = {v4[it].x, v4[it].y, v4[it].z, v4[it].w};
            uint32_t bits = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool take = v[j] >= least && v[j] != -INFINITY;
                picks |= take ? 1u << (4 * it + j) : 0u;
                if (TAILS) {
                    const uint32_t f = small31((v[j] - r.top) * r.c_hi);
                    bits += take || v[j] == -INFINITY ? 0u : f;
                }
            }
            if (TAILS) tail += bits;
        }
        if (picks) {
            int at = atomicAdd(&sh->picked, __popc(picks));
            for (; picks; picks &= picks - 1, ++at) {
                const int bit = __ffs(picks) - 1, i = base0 + (bit >> 2) * 4 * kSampleThreads + (bit & 3);
                if (at < kPickMax) sh->pick[at] = i;
            }
        }
    }
    __syncthreads();
    const int n = min(sh->picked, kPickMax);
    for (int j = tid; j < n; j += kSampleThreads) sh->pick_l[j] = r.at(sh->pick[j]);      // (each thread reads its own later)
    return tail;
}
// f(token, its logit) for the picked tokens
template <typename T, typename F>
__device__ __forceinline__ void for_picked(SampleShared* sh, const Row<T>& r, float least, F f) {
    const int n = sh->picked;
    if (n <= kPickMax) {
        for (int j = threadIdx.x; j < n; j += kSampleThreads) f(sh->pick[j], sh->pick_l[j]);
    } else {
        constexpr int kFlight = 2;                       // vectors of a thread on their way
        for (int base = 4 * threadIdx.x; base < r.n; base += 4 * kFlight * kSampleThreads) {
            float4 x[kFlight];
#pragma unroll
            for (int it = 0; it < kFlight; ++it) x[it] = r.four(base + it * 4 * kSampleThreads);
#pragma unroll 1
            for (int it = 0; it < kFlight; ++it) {
                const float4 v = x[0];
#pragma unroll
                for (int k = 0; k + 1 < kFlight; ++k) x[k] = x[k + 1];
                const int i = base + it * 4 * kSampleThreads;
                if (v.x >= least && v.x != -INFINITY) f(i, v.x);
                if (v.y >= least && v.y != -INFINITY) f(i + 1, v.y);
                if (v.z >= least && v.z != -INFINITY) f(i + 2, v.z);
                if (v.w >= least && v.w != -INFINITY) f(i + 3, v.w);
            }
        }
    }
}

__device__ __forceinline__ u64 share_of(u64 whole, double share) { return min(whole, max((u64)1, (u64)ceil((double)whole * share))); }
// Sums of the block's warps before this one, from `sums` (a warp each), and of all.
__device__ __forceinline__ u64 warps_before(const u64* sums, u64& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const u64 own = lane < kSampleWarps ? sums[lane] : 0, in = warp_scan(own, lane);
    total = __shfl_sync(0xffffffffu, in, 31);
    return __shfl_sync(0xffffffffu, in - own, warp);
}

// Blocks of a row: all meet, shared memory of any of them.
struct Blocks {
    int n, rank;
    __device__ __forceinline__ void sync() const {
        if (n == 1) __syncthreads();
        else cg::this_cluster().sync();
    }
    __device__ __forceinline__ void leave() const {
        if (n == 1) return;
        __syncwarp();                                     // lanes come from loops of different trips; the barrier is the warp's
        asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    }
    __device__ __forceinline__ SampleShared* at(SampleShared* sh, int r) const { return n == 1 ? sh : cg::this_cluster().map_shared_rank(sh, r); }
};

__device__ __forceinline__ void clear_steps(SampleShared* sh) {
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { sh->lo[i] = 0; sh->hi[i] = 0; }
    if (threadIdx.x == 0) sh->tail = 0;
    __syncthreads();
}
// (other blocks read the steps and the list's length: not before they have met)
__device__ __forceinline__ void clear_pass(SampleShared* sh) {
    if (threadIdx.x == 0) { sh->list_n = 0; sh->range_lo = ~0ull; sh->range_hi = 0; }
    clear_steps(sh);
}

// The step in which the sum over steps passes the target, over all blocks' histograms; every block finds the same.  The target
// is `target`, or with share >= 0 that part of the whole sum.  Written to sh->bin (kBins: beyond the steps), sh->before, sh->target.
__device__ void find_bin(SampleShared* sh, const Blocks& blocks, u64 start, u64 target, double share) {
    blocks.sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    u64 v0 = 0, v1 = 0, tail = 0;
    for (int r = 0; r < blocks.n; ++r) {
        const SampleShared* o = blocks.at(sh, r);
        const uint2 lo = *reinterpret_cast<const uint2*>(&o->lo[2 * tid]), hi = *reinterpret_cast<const uint2*>(&o->hi[2 * tid]);
        v0 += ((u64)hi.x << 32) + lo.x;
        v1 += ((u64)hi.y << 32) + lo.y;
        tail += o->tail;
    }
    u64 in = warp_scan(v0 + v1, lane);
    if (lane == 31) sh->scan[warp] = in;
    __syncthreads();
    u64 total;
    in += start + warps_before(sh->scan, total);
    if (tid == 0) {
        sh->bin = kBins;
        sh->target = share >= 0.0 ? share_of(start + total + tail, share) : target;
    }
    __syncthreads();
    target = sh->target;
    const u64 mid = in - v1;
    if (mid - v0 < target && target <= mid) { sh->bin = 2 * tid; sh->before = mid - v0; }
    if (mid < target && target <= in) { sh->bin = 2 * tid + 1; sh->before = mid; }
    __syncthreads();      // (other blocks may still read this block's histogram: its next change comes behind another meeting)
}

// On a short list (n at most kShort, by its block alone) every token is compared with every other: the first `count` of them in the
// order are kept, and of those the ones before which the sum, `before` included, is below the target: `target`, or with share >= 0
// that part of their sum.  Written to sh->cut.
constexpr int kShort = 256;
__device__ void short_list(SampleShared* sh, const Scale& r, int n, u64 before, u64 target, u64 count, double share) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __syncthreads();
    const u64 p = tid < n ? sh->list[tid] : ~0ull;
    const uint32_t f = tid < n ? mass31(r, logit_at(p)) : 0u;
    if (tid < n) sh->lo[tid] = f;
    __syncthreads();
    u64 sum = 0;
    uint32_t rank = 0;
    if (tid < n) {
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const bool earlier = sh->list[j] < p;
            rank += earlier;
            sum += earlier ? sh->lo[j] : 0u;
        }
    }
    const bool keep = tid < n && (u64)rank < count;
    if (share >= 0.0) {
        u64 all = keep ? f : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        if (lane == 0) sh->scan[warp] = all;
        __syncthreads();
        warps_before(sh->scan, all);
        if (tid == 0) sh->target = share_of(before + all, share);
        __syncthreads();
        target = sh->target;
    }
    sum += before;
    // the last token kept: nothing kept behind it
    const bool in = keep && sum < target;
    if (in && ((u64)rank + 1 == min((u64)n, count) || sum + f >= target)) sh->cut = p;
    __syncthreads();
}

// The cut of the first block's list of n places (by that block alone): the place at which the sum of f (MASS) or the count, over
// places up to `limit` and from `before` on, reaches the target.  Written to sh->cut.
template <bool MASS>
__device__ void list_cut(SampleShared* sh, const Scale& r, int n, u64 before, u64 target, u64 limit) {
    const int tid = threadIdx.x, lane = tid & 31;
    const Blocks alone{1, 0};
    if (MASS && n <= kShort && limit == ~0ull) {
        short_list(sh, r, n, before, target, ~0ull, -1.0);
        return;
    }
    u64 lo = ~0ull, hi = 0;
    __syncthreads();
    if (tid == 0) { sh->range_lo = ~0ull; sh->range_hi = 0; sh->few_n = 0; }
    __syncthreads();
    for (int i = tid; i < n; i += kSampleThreads) {
        const u64 p = sh->list[i];
        if (p <= limit) { lo = min(lo, p); hi = max(hi, p); }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    if (lane == 0) { atomicMin(&sh->range_lo, lo); atomicMax(&sh->range_hi, hi); }
    __syncthreads();
    lo = sh->range_lo;
    hi = sh->range_hi;
    for (;;) {
        for (int i = tid; i < n; i += kSampleThreads) {
            const u64 p = sh->list[i];
            if (p < lo || p > hi) continue;
            const int at = atomicAdd(&sh->few_n, 1);
            if (at < 32) sh->few[at] = p;
        }
        __syncthreads();
        const int m = sh->few_n;
        if (m <= 32) {
            if (tid < 32) {
                const u64 p = lane < m ? sh->few[lane] : ~0ull;
                const uint32_t f = lane < m ? (MASS ? mass31(r, logit_at(p)) : 1u) : 0u;
                u64 sum = before;
                for (int j = 0; j < m; ++j) {
                    const u64 pj = __shfl_sync(0xffffffffu, p, j);
                    const uint32_t fj = __shfl_sync(0xffffffffu, f, j);
                    if (pj < p) sum += fj;
                }
                if (lane < m && sum < target && target <= sum + f) sh->cut = p;
            }
            __syncthreads();
            return;
        }
        int shift = 0;
        while (((hi - lo) >> shift) >= (u64)kBins) ++shift;
        clear_steps(sh);
        for (int i = tid; i < n; i += kSampleThreads) {
            const u64 p = sh->list[i];
            if (p >= lo && p <= hi) hist_add<MASS>(sh, (int)((p - lo) >> shift), MASS ? mass31(r, logit_at(p)) : 0u);
        }
        find_bin(sh, alone, before, target, -1.0);
        before = sh->before;
        lo += (u64)sh->bin << shift;
        hi = min(hi, lo + (((u64)1 << shift) - 1));
        if (tid == 0) sh->few_n = 0;
        __syncthreads();
    }
}
// Both filters on a list that holds every token they keep: the first `count` of it, then, with share >= 0, that part of their mass.
__device__ void list_filters(SampleShared* sh, const Scale& r, int n, u64 count, double share) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (n <= kShort) {
        short_list(sh, r, n, 0, ~0ull, count, share);
        return;
    }
    list_cut<false>(sh, r, n, 0, count, ~0ull);
    if (share < 0.0) return;
    const u64 limit = sh->cut;
    u64 sum = 0;
    for (int i = tid; i < n; i += kSampleThreads) {
        const u64 p = sh->list[i];
        if (p <= limit) sum += mass31(r, logit_at(p));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();
    if (lane == 0) sh->scan[warp] = sum;
    __syncthreads();
    u64 total;
    warps_before(sh->scan, total);
    if (tid == 0) sh->target = share_of(total, share);
    __syncthreads();
    list_cut<true>(sh, r, n, 0, sh->target, limit);
}

// Collects the picked tokens for which `take` says so in the first block's list; returns how many there are (the list holds
// kListMax).
template <typename T, typename F>
__device__ __forceinline__ int collect(SampleShared* sh, const Blocks& blocks, const Row<T>& r, float least, F take) {
    SampleShared* first = blocks.at(sh, 0);
    u64 mn = ~0ull, mx = 0;
    for_picked(sh, r, least, [&](int i, float l) {
        if (!take(l, i)) return;
        const u64 p = place_of(l, r.first + i);
        mn = min(mn, p);
        mx = max(mx, p);
        const int at = atomicAdd(&first->list_n, 1);
        if (at < kListMax) first->list[at] = p;
    });
    if (mn != ~0ull) { atomicMin(&sh->range_lo, mn); atomicMax(&sh->range_hi, mx); }
    blocks.sync();
    return first->list_n;
}

// Where more tokens lie above 2^-kTail of the largest than are listed: the highest of 2^-10, 2^-11 .. below which there is less than
// what top-p leaves out (by a margin that covers the rounding of this count), so that the cut lies above.  All blocks find the same.
template <typename T>
__device__ float higher_tail(SampleShared* sh, const Blocks& blocks, const Row<T>& r, double share) {
    const int tid = threadIdx.x, lane = tid & 31;
    __syncthreads();
    if (tid <= kSteps) sh->below[tid] = 0;
    __syncthreads();
    uint32_t sum[kSteps + 1] = {};
    for (int base = 4 * tid; base < r.n; base += 16 * kSampleThreads) {
        float4 v4[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) v4[it] = r.four(base + it * 4 * kSampleThreads);
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const float v[4] = {v4[it].x, v4[it].y, v4[it].z, v4[it].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e = v[j] == r.top ? 0.0f : (v[j] - r.top) * r.c_hi;
                float w;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(e));
                const uint32_t f = v[j] == -INFINITY ? 0u : (uint32_t)(__float_as_int(fmaf(w, 1048576.0f, 12582912.0f)) - 0x4B400000);
                sum[kSteps] += f;
#pragma unroll
                for (int k = 0; k < kSteps; ++k) sum[k] += e < -(kTail - kSteps + k) ? f : 0u;
            }
        }
    }
#pragma unroll
    for (int k = 0; k <= kSteps; ++k) {
        u64 x = sum[k];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (lane == 0 && x) atomicAdd(&sh->below[k], x);
    }
    blocks.sync();
    u64 below[kSteps + 1] = {};
    for (int q = 0; q < blocks.n; ++q)
#pragma unroll
        for (int k = 0; k <= kSteps; ++k) below[k] += blocks.at(sh, q)->below[k];
    if (tid == 0) {
        float tail = kTail;
        const double round = 0.5 * (double)r.whole, out = (1.0 - share) * ((double)below[kSteps] - round) * 0.999;
#pragma unroll
        for (int k = kSteps - 1; k >= 0; --k)
            if ((double)below[k] + round < out) tail = kTail - kSteps + k;
        sh->red[0] = r.top - tail / r.c_hi;
    }
    __syncthreads();
    return sh->red[0];
}

// The cut: the token at which the sum of weights (MASS) or the count over the order passes the target: `target`, or with
// share >= 0 that part of the whole.  `limit` is a cut found before: tokens behind it do not take part.  The picked tokens (those
// from `least` on) hold the cut; with `tails` that is not known yet, and `least` may be lowered.  The first block has the result,
// before the next meeting.
template <bool MASS, typename T>
__device__ void select_cut(SampleShared* sh, const Blocks& blocks, const Row<T>& r, u64 target, double share, u64 limit, bool tails,
                           float& least) {
    const int lane = threadIdx.x & 31;
    bool again = false;
    for (;;) {
        clear_pass(sh);
        if (tails) {
            u64 tail = pick_tokens<true, T>(sh, r, least);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) tail += __shfl_xor_sync(0xffffffffu, tail, o);
            if (lane == 0 && tail) atomicAdd(&sh->tail, tail);
        }
        bool counted = false, anew = false;
        for (;;) {
            const bool survey = tails && !again;
            if (!counted && (!survey || sh->picked <= kPickMax)) {
                for_picked(sh, r, least, [&](int i, float l) {
                    if (limit != ~0ull && place_of(l, r.first + i) > limit) return;
                    hist_add<MASS>(sh, bin_of(r, l), MASS ? mass31(r, l) : 0u);
                });
                counted = true;
            }
            find_bin(sh, blocks, 0, target, share);
            if (!survey) break;
            again = true;
            int picked = 0;
            for (int q = 0; q < blocks.n; ++q) picked = max(picked, blocks.at(sh, q)->picked);
            if (picked <= kPickMax) break;
            const float higher = higher_tail(sh, blocks, r, share);
            if (higher > least) {
                least = higher;
                anew = true;
                break;
            }
        }
        if (anew) continue;
        if (sh->bin < kBins || !tails) break;
        blocks.sync();                                   // (all have read the others' counts)
        least = -INFINITY;                               // among the small ones: all tokens, exactly
        tails = false;
        pick_tokens<false, T>(sh, r, least);
        blocks.sync();
    }
    target = sh->target;
    const int bin = sh->bin;
    u64 before = sh->before, lo = 0, hi = ~0ull;
    for (;;) {
        const int n = collect(sh, blocks, r, least, [&](float l, int i) {
            if (bin_of(r, l) != bin) return false;
            const u64 p = place_of(l, r.first + i);
            return p <= limit && p >= lo && p <= hi;
        });
        if (n <= kListMax) {
            if (blocks.rank == 0) list_cut<MASS>(sh, r, n, before, target, ~0ull);
            return;
        }
        // too many: split the range of places
        u64 a = ~0ull, z = 0;
        for (int k = 0; k < blocks.n; ++k) {
            const SampleShared* o = blocks.at(sh, k);
            a = min(a, o->range_lo);
            z = max(z, o->range_hi);
        }
        blocks.sync();
        int shift = 0;
        while (((z - a) >> shift) >= (u64)kBins) ++shift;
        clear_pass(sh);
        for_picked(sh, r, least, [&](int i, float l) {
            if (bin_of(r, l) != bin) return;
            const u64 p = place_of(l, r.first + i);
            if (p > limit || p < a || p > z) return;
            hist_add<MASS>(sh, (int)((p - a) >> shift), MASS ? mass31(r, l) : 0u);
        });
        find_bin(sh, blocks, before, target, -1.0);
        before = sh->before;
        lo = a + ((u64)sh->bin << shift);
        hi = min(z, lo + (((u64)1 << shift) - 1));
        blocks.sync();
        clear_pass(sh);                                                       // the list starts anew
        blocks.sync();
    }
}

// grid: rows * cluster size
template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
    extern __shared__ float4 raw4[];
    SampleShared* sh = reinterpret_cast<SampleShared*>(raw4);
    Blocks blocks;
    blocks.n = (int)cg::this_cluster().num_blocks();
    blocks.rank = (int)cg::this_cluster().block_rank();
    const int rank = blocks.rank;
    const long long row = blockIdx.x / blocks.n;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int first = rank * a.segment, n = max(0, min(a.segment, a.V - first));
    const T* src = static_cast<const T*>(a.logits) + row * a.row_stride + first;

    const float T_in = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = !(T_in > 0.0f);
    if (tid == kSampleThreads - 1) {
        const double t = greedy ? 1.0 : (double)T_in, inv = 1.4426950408889634 / t;
        sh->c_hi = (float)fmin(inv, 1e38);               // a temperature near zero: finite, so that the top keeps weight 1
        sh->c_lo = inv < 1e38 ? (float)(inv - (double)sh->c_hi) : 0.0f;
        sh->bin_scale = fminf((float)((double)kBins / (kBinSpan * t)), 1e30f);
    }
    // ---- the row's largest logit, and how many are not -infinity (NaN counts as that)
    Row<T> r;
    r.data = src; r.n = n; r.first = first; r.whole = a.V; r.vec = a.vec_in;
    const float u_first = a.tokens && warp < a.K ? a.u[row * a.K + warp] : 0.0f;      // the warp's first draw
    float mine = -INFINITY;
    int live = 0;
    for (int base = 4 * tid; base < n; base += 32 * kSampleThreads) {
        float4 v[8];
#pragma unroll
        for (int it = 0; it < 8; ++it) v[it] = r.four(base + it * 4 * kSampleThreads);
#pragma unroll
        for (int it = 0; it < 8; ++it) {
            mine = fmaxf(mine, fmaxf(fmaxf(v[it].x, v[it].y), fmaxf(v[it].z, v[it].w)));
            live += (v[it].x != -INFINITY) + (v[it].y != -INFINITY) + (v[it].z != -INFINITY) + (v[it].w != -INFINITY);
        }
    }
    const int padded = (n + kChunk - 1) / kChunk * kChunk;
    float mx = mine;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    live = __reduce_add_sync(0xffffffffu, live);
    if (lane == 0) { sh->red[warp] = mx; sh->red_live[warp] = live; }
    __syncthreads();
    if (warp == 0) {
        float v = lane < kSampleWarps ? sh->red[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        const int c = __reduce_add_sync(0xffffffffu, lane < kSampleWarps ? sh->red_live[lane] : 0);
        if (lane == 0) { sh->block_max = v; sh->block_live = c; }
    }
    blocks.sync();
    float top = -INFINITY;
    live = 0;
    for (int k = 0; k < blocks.n; ++k) {
        const SampleShared* o = blocks.at(sh, k);
        top = fmaxf(top, o->block_max);
        live += o->block_live;
    }

    // ---- the filters of this row
    r.top = top;
    r.c_hi = sh->c_hi; r.c_lo = sh->c_lo; r.bin_scale = sh->bin_scale;
    int k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
    if (k < 0 || k >= live) k = 0;                       // off
    const float tp = greedy || !a.top_p ? 1.0f : a.top_p[row], mp = greedy || !a.min_p ? 0.0f : a.min_p[row];
    const double share = tp < 1.0f ? (double)fmaxf(tp, 0.0f) : -1.0;
    float* dst = a.probs ? a.probs + row * a.V + first : nullptr;
    const bool sparse = top > -INFINITY && (k > 0 || share >= 0.0);      // what is kept are some of the picked tokens
    u64 cut = ~0ull;
    float least = -INFINITY;
    if (sparse) {
        bool found = false;
        if (k > 0) {
            clear_pass(sh);
            if (2 * k <= blocks.n * kSampleThreads) {    // by the threads' maxima, or by those of four tokens
                if (mine != -INFINITY) atomicAdd(&sh->lo[bin_of(r, mine)], 1u);
            } else {
                for (int base = 4 * tid; base < n; base += 16 * kSampleThreads) {
                    float4 v[4];
#pragma unroll
                    for (int it = 0; it < 4; ++it) v[it] = r.four(base + it * 4 * kSampleThreads);
#pragma unroll
                    for (int it = 0; it < 4; ++it) {
                        const float m = fmaxf(fmaxf(v[it].x, v[it].y), fmaxf(v[it].z, v[it].w));
                        if (m != -INFINITY) atomicAdd(&sh->lo[bin_of(r, m)], 1u);
                    }
                }
            }
            find_bin(sh, blocks, 0, (u64)k, -1.0);
            const int step = sh->bin;                    // kBins where there are fewer than k maxima
            least = step_floor(r, step);
            pick_tokens<false, T>(sh, r, least);
            if (k <= kListK && step < kBins) {
                const int got = collect(sh, blocks, r, least, [&](float l, int) { return bin_of(r, l) <= step; });
                found = got <= kListMax;
                if (found && rank == 0) list_filters(sh, r, got, (u64)k, share);
            }
            if (!found) {
                blocks.sync();                           // all have seen it: the list may start anew
                select_cut<false>(sh, blocks, r, (u64)k, -1.0, ~0ull, false, least);
                blocks.sync();
                cut = blocks.at(sh, 0)->cut;
            }
        }
        if (!found && share >= 0.0) {
            blocks.sync();
            if (k == 0) {
                least = r.top - kTail / r.c_hi;
                if (!(least > -INFINITY)) least = -INFINITY;
                if (top == INFINITY) least = INFINITY;   // nothing else carries mass
            }
            select_cut<true>(sh, blocks, r, 0, share, cut, k == 0, least);
        }
        blocks.sync();
        cut = blocks.at(sh, 0)->cut;
        if (sh->picked > kPickMax && cut != ~0ull) pick_tokens<false, T>(sh, r, logit_at(cut));   // what is kept may be few
        __syncthreads();
    }

    // ---- weights of what is kept, and their sums by chunks of 128
    const float floor_w = mp > 0.0f ? fminf(mp, 1.0f) : 0.0f;
    const int chunks = padded / kChunk;
    const bool listed = sparse && sh->picked <= kPickMax;
    const float cut_l = cut != ~0ull ? logit_at(cut) : -INFINITY;
    const uint32_t cut_id = (uint32_t)cut;               // with -infinity: none is kept there
    auto kept_weight = [&](float l, int i) -> float {
        if (l == -INFINITY || l < cut_l || (l == cut_l && (uint32_t)(first + i) > cut_id)) return 0.0f;
        const float w = weight(r, l);
        return w < floor_w ? 0.0f : w;
    };
    auto weights_of = [&](float4 v, int i) -> float4 {
        return make_float4(kept_weight(v.x, i), kept_weight(v.y, i + 1), kept_weight(v.z, i + 2), kept_weight(v.w, i + 3));
    };
    auto four_weights = [&](int i) -> float4 { return weights_of(r.four(i), i); };
    if (listed) {
        for (int i = tid; i <= chunks; i += kSampleThreads) sh->chunk[i] = 0;
        __syncthreads();
        for (int j = tid; j < sh->picked; j += kSampleThreads) {
            const int i = sh->pick[j];
            const float w = kept_weight(sh->pick_l[j], i);
            sh->pick_l[j] = w;
            if (w > 0.0f) atomicAdd(&sh->chunk[i / kChunk + 1], (u64)fixed31(w));
        }
    } else {
        __syncthreads();
        for (int c0 = warp; c0 < chunks; c0 += 4 * kSampleWarps) {
            float4 x[4];
#pragma unroll
            for (int it = 0; it < 4; ++it) x[it] = r.four((c0 + it * kSampleWarps) * kChunk + lane * 4);
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int c = c0 + it * kSampleWarps;
                if (c >= chunks) break;
                const float4 v = weights_of(x[it], c * kChunk + lane * 4);
                const uint32_t f0 = fixed31(v.x), f1 = fixed31(v.y), f2 = fixed31(v.z), f3 = fixed31(v.w);
                const uint32_t hi = __reduce_add_sync(0xffffffffu, (f0 >> 16) + (f1 >> 16) + (f2 >> 16) + (f3 >> 16));
                const uint32_t lo = __reduce_add_sync(0xffffffffu, (f0 & 0xffffu) + (f1 & 0xffffu) + (f2 & 0xffffu) + (f3 & 0xffffu));
                if (lane == 0) sh->chunk[c + 1] = ((u64)hi << 16) + lo;
            }
        }
    }
    __syncthreads();
    if (warp == 0) {                                     // running sums of the chunks
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
    blocks.sync();
    u64 all = 0, mine0 = 0;
    for (int q = 0; q < blocks.n; ++q) {
        const u64 t = blocks.at(sh, q)->total;
        if (q < rank) mine0 += t;
        all += t;
    }
    const u64 mine1 = mine0 + sh->total;
    if (tid == kSampleThreads - 1) sh->scale = all ? (float)(2147483648.0 / (double)all) : 0.0f;
    __syncthreads();

    // ---- draws: the first token at which the running sum passes u * sum
    if (a.tokens) {
        for (int j = warp; j < a.K; j += kSampleWarps) {
            int32_t* out = a.tokens + row * a.K + j;
            if (all == 0) {                              // no token left: every logit is -infinity or NaN
                if (rank == 0 && lane == 0) *out = -1;
                continue;
            }
            u64 t = 0;
            if (lane == 0) {
                const double x = (double)(j < kSampleWarps ? u_first : a.u[row * a.K + j]) * (double)all;
                if (x > 0.0) t = min(all - 1, (u64)x);
            }
            t = __shfl_sync(0xffffffffu, t, 0);
            if (t < mine0 || t >= mine1) continue;       // another block's
            const u64 at = t - mine0;
            int lo = 0, hi = chunks;                     // chunk[lo] <= at < chunk[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sh->chunk[mid] <= at) lo = mid; else hi = mid;
            }
            const float4 v = four_weights(lo * kChunk + lane * 4);
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
    if (dst) {
        const float scale = sh->scale;
        if (listed) {                                    // zeros, and the few values between them
            if (a.vec_out) {
                for (int i = tid * 4; i < n; i += kSampleThreads * 4) __stcs(reinterpret_cast<float4*>(dst + i), make_float4(0.0f, 0.0f, 0.0f, 0.0f));
            } else {
                for (int i = tid; i < n; i += kSampleThreads) __stcs(dst + i, 0.0f);
            }
            __syncthreads();
            for (int j = tid; j < sh->picked; j += kSampleThreads)
                if (sh->pick_l[j] > 0.0f) __stcs(dst + sh->pick[j], sh->pick_l[j] * scale);
        } else if (a.vec_out) {
            for (int i0 = tid * 4; i0 < n; i0 += 16 * kSampleThreads) {
                float4 x[4];
#pragma unroll
                for (int it = 0; it < 4; ++it) x[it] = r.four(i0 + it * 4 * kSampleThreads);
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int i = i0 + it * 4 * kSampleThreads;
                    if (i >= n) break;
                    float4 v = weights_of(x[it], i);
                    v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
                    __stcs(reinterpret_cast<float4*>(dst + i), v);
                }
            }
        } else {
            for (int i = tid; i < n; i += kSampleThreads) __stcs(dst + i, kept_weight(r.at(i), i) * scale);
        }
    }
    blocks.leave();                                      // no block leaves while another may read its shared memory
}

}  // namespace mcsd

extern "C" int mcsd_sample_candidates(const void* logits, long long row_stride, int dtype, int rows, int V, const float* temperature,
                                      const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int K,
                                      int32_t* tokens, float* probs, void* stream) {
    if (!logits || (!tokens && !probs) || (tokens && !u)) return MCSD_ERR_NULL;
    if (dtype != MCSD_BF16 && dtype != MCSD_F32) return MCSD_ERR_BAD_DTYPE;
    if (rows < 1 || rows > (1 << 24) || V < 1 || V > mcsd::kSampleMaxVocab || row_stride < V || K < 0 || (tokens && (K < 1 || K > 1024)))
        return MCSD_ERR_BAD_SHAPE;
    int dev = 0, sms = 0;
    MCSD_CUDA_CHECK(cudaGetDevice(&dev));
    MCSD_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // blocks a row: more while there are multiprocessors without a row (a block of 1024 tokens is mostly meetings), and a second
    // block on each where a block keeps 16384 (100 rows of 131072: 43 or 49 us with top-k, 52 or 118 with top-p)
    int c = 1;
    while (c < 8 && ((long long)rows * c * 2 <= sms && V / (c * 2) >= 1024 || (long long)rows * c <= sms && V / (c * 2) >= 16384)) c *= 2;
    mcsd::SampleArgs a{};
    a.logits = logits; a.row_stride = row_stride;
    a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u;
    a.tokens = tokens; a.probs = probs;
    a.V = V; a.K = K;
    a.segment = ((V + c - 1) / c + mcsd::kChunk - 1) / mcsd::kChunk * mcsd::kChunk;
    const int elt = dtype == MCSD_F32 ? 4 : 2;
    a.vec_in = (reinterpret_cast<uintptr_t>(logits) & 15u) == 0 && (row_stride * elt) % 16 == 0;
    a.vec_out = probs && (reinterpret_cast<uintptr_t>(probs) & 15u) == 0 && V % 4 == 0;
    const int smem = (int)sizeof(mcsd::SampleShared);
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
