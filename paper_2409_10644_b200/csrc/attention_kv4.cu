// Tree attention (Section 2.2 of the paper) over a prefix cache held in 4 bits (page layout in kv4.cuh), on the
// fifth-generation tensor cores of sm_100a: bf16 tree tensors, head_dim 128, 1 to 64 query columns per work item.
//
// The products are set up transposed, the small dimension (query columns) as the MMA N:
//     S^T[key][query] = K Q^T,     O^T[channel][query] += V^T P^T,     l[query] += P 1
// and the A operands of the first two live in tensor memory, not in shared memory: thread r of the key warps owns key row r of a
// 128-key tile, thread d of the value warps channel d, and both turn 16-byte pieces of a page (neighbouring threads read
// neighbouring pieces) into operand columns with a shift and a mask per two values and store them with tcgen05.st.
//   * Keys stay codes: the byte c (0..15) is c 2^-9 in e4m3 (its two lowest binades have the same spacing), so eight codes
//     become operands with two masks and a shift.  Queries are split into two e4m3 parts, high and low, on a power of two common to
//     the work item that brings its largest to 128 .. 256: together they hold all eight bits of a bf16 number down to 2^-9 of
//     the largest, and what is smaller to within 2^-17 of the largest.  That is 2^-14 of a row's own largest or less while no
//     row's largest lies further than a factor of 8 below the item's.  Where one does, so that a row would suffer from its
//     neighbours, the item's codes become bf16 numbers 16 + c against the bf16 queries (no rounding; the keys of a tile
//     then take both buffers, as the tree's do: 180 us against 160 for the 45-node trees, 92 against 68 for long single tokens,
//     467 against 348 for the forests).  The sums are exact up to fp32, and the row's scale and offset are applied to
//     the score, where the softmax thread owns the same key row:
//         score = scale_k (sum of code q) + (16 scale_k + offset_k) (sum of q).
//   * Values become scale_v (16 + code) + offset_v, one packed fused multiply-add per two values.  They and the weights
//     that multiply them are fp16 (11 bits: an order of magnitude below the rounding of the bf16 result) in every tile
//     whose values and weights both lie well inside fp16's range, which the key warps vote on for the values and the softmax
//     group for the weights; else both are bf16 (8 bits, as in the kernel over dense caches).  A tile whose weights say so late
//     has its values converted in tensor memory: 235 us against 160 for the 45-node trees, 84 against 68 for long single tokens,
//     with scores three times as large (a standard deviation of 4 nats).
// The rows of the tree itself are read as they are (bf16, against the bf16 queries): scale 1, offset 0.
//
// What bounds it: 136 bytes per key and head against 512 in bf16 move the floor of a launch down by 3.8; unpacking
// and the exponentials then share the issue slots of the schedulers, so the work is spread over specialised warps:
//   warps 0-3    keys      page pieces -> operand columns, and the scales of the value rows
//   warps 4-11   values    page pieces -> operand columns; warps 4-7 the even tiles, 8-11 the odd ones
//   warps 12-19  softmax   warps 12-15 the even tiles, 16-19 the odd ones.  The two groups have their own references,
//                accumulators and row sums and meet only at the end of a work item: a tile's chain (scores, exponentials, vote,
//                P^T, products) may take twice the time between two tiles
//   warp 20      copies whole pages (1 to 4 of them, contiguous) into a ring with cp.async.bulk
//   warps 21, 22 issue the MMAs of the scores and of the products
//   warp 23      brings the queries of the next work item and their sums
// Loops are rolled as far as the latencies allow: the roles share the instruction caches, and with unrolled bodies (a
// kernel of 180 KB) a tile took three times as long, most of it in waits for instructions.
//
// Work: one block per multiprocessor walks a contiguous range of the (sequence, key/value head, query block, tile) space,
// cut by cost.  A work item that a range boundary cuts is finished by whichever of its blocks comes last (a counter of
// tiles per item; nothing waits): it reads all pieces in block order, so the result does not depend on who that is.
// Every wait is bounded; one that runs out raises a flag in the workspace header.
//
// Measured (whole calls back to back): 16 sequences of 4096 rows, 32 heads, 45-node trees: 160 us, 1.9 TB/s (the bytes alone take
// 47 us at the copy rate); 8 sequences up to 32001 rows, 8 key/value heads, one token: 68 us, 2.4 TB/s (25 us); 32 ragged
// sequences with 8 to 160 nodes, one to three query blocks each: 349 us (58 us).  Against the kernel over dense bf16 caches
// (events, cold cache): 169 / 75 / 352 us here, 179 / 116 / 286 us there, so with many nodes the cache's size is the gain, not
// the time.  Counters: 52 % of the issue slots used with six warps per scheduler on the trees (19 % of the memory's rate), 49 % on
// the long tokens (27 %); the warps wait for one another's barriers, and for instructions.  Tried and slower: both halves of a
// tile's columns on groups of their own (28 and more warps, 64 registers), a second buffer for P^T, longer unrolled loops; and
// warp-level matrix instructions on operands unpacked into registers (324 us for the 45-node trees).
#include <algorithm>
#include <mutex>
#include <type_traits>

#include <cuda_fp16.h>

#include "attention_tc_common.cuh"
#include "f32x2.cuh"
#include "kv4.cuh"

namespace mcsd {

namespace {

constexpr int kD = 128;
constexpr int kPageBytes = kv4_page_bytes(kD);
constexpr int kStageBytes = 4 * kPageBytes;      // one tile: 128 rows
constexpr int kValueWarp = 4, kSoftWarp = 12, kCopyWarp = 20, kScoreWarp = 21, kProductWarp = 22, kQueryWarp = 23;
constexpr int kThreads = 32 * (kQueryWarp + 1), kSoftThreads = 256;
constexpr int kWideQ = 64;                       // query columns of a work item, at most
template <int QB> constexpr int kStages = QB > 16 ? 5 : 6;   // tiles of codes in the ring: what fits
// Tensor-memory columns: scores, O^T and row sums of the two softmax groups (the sums with a query per lane and sixteen identical
// columns, of which the first counts), keys (two buffers of codes; a tile of tree rows takes
// both), values.
template <int QB>
struct Columns {
    static constexpr int S = 0, O = 2 * QB, L = 4 * QB, K = L + 32, V = K + 64;
    static_assert(V + 128 <= kTmemCols, "tensor memory");
};

struct Params {
    const __nv_bfloat16 *q, *k_tree, *v_tree;
    const unsigned char* cache;
    __nv_bfloat16* out;
    const int32_t *seq_lens, *n_active;
    const uint64_t* anc;
    int words, B, Hkv, G, N, pages;
    float scale_log2;
    float* part_ml;       // [2 * kMaxCtas][2][kWideQ]
    float* part_o;        // [2 * kMaxCtas][kWideQ][128]
    int* counters;        // [blocks][kCountersPerBlock], the first: finished tiles of the cut work item that the block starts; zero between launches
    WorkspaceHeader* header;
};

// Per-sequence tables, the same in every block.
struct Plan {
    long long tiles[kMaxBatchTc + 1], cost[kMaxBatchTc + 1];   // of the sequences before b
    int items[kMaxBatchTc + 1];
    int len[kMaxBatchTc], nodes[kMaxBatchTc];
    long long first[kMaxCtas + 1];   // first tile of every block
    int blocks;
};

// Cost of a tile with nq query columns (unpacking bounds it up to 16 columns, the exponentials beyond: about 29 cycles per unit)
// and of a work item on top of its tiles: its queries, first references, the tree rows read as they are, its end.  Measured on
// 32 ragged sequences with 8 to 160 nodes / the 45-node trees / 8 long single tokens: 349 / 160 / 68 us with 400, 377 / 161 / 67
// with 256, 393 / 162 / 66 with 200, 430 / 163 / 66 with 100.
__host__ __device__ __forceinline__ int tile_cost(int nq) { return nq < 16 ? 40 : 24 + nq; }
constexpr int kItemCost = 400;

// Weights are 2^(score - reference).  A reference is taken 2^kFirstLog below the score it comes from and raised when a weight
// passes 2^kTopLog; fp16 keeps the relative precision of what lies between 2^kLowLog and 2^kTopLog.  A lower first reference
// leaves more room for small weights and is raised more often: 160 us for the 45-node trees with 4 to 6, 166 with 8, 180 with 10.
constexpr float kFirstLog = 5.f, kTopLog = 15.f, kLowLog = -14.f;

struct Shape {            // of the work items of one sequence
    int Tp, T, blocks_q, per_q, total_q;
};
template <int QB>
__host__ __device__ __forceinline__ Shape shape_of(int L, int Nb, int G) {
    Shape s;
    s.total_q = Nb * G;
    s.blocks_q = (s.total_q + QB - 1) / QB;
    s.per_q = s.blocks_q ? ((s.total_q + s.blocks_q - 1) / s.blocks_q + 7) & ~7 : 0;
    s.Tp = (L + kTile - 1) / kTile;
    s.T = Nb > 0 ? s.Tp + (Nb + kTile - 1) / kTile : 0;
    return s;
}

struct Piece {            // the tiles of one work item that a block takes
    int b, hk, item, lt, T, Tp, L, Nb, q0, Nq;
    int cnt;
};

template <int QB>
__device__ __forceinline__ void piece_at(const Plan& pl, const Params& p, long long t, long long t_end, Piece& s) {
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pl.tiles[mid] <= t) lo = mid; else hi = mid;
    }
    s.b = lo;
    s.L = pl.len[lo];
    s.Nb = pl.nodes[lo];
    const Shape sh = shape_of<QB>(s.L, s.Nb, p.G);
    const uint32_t r = (uint32_t)(t - pl.tiles[lo]);          // below 2^31 by the limit on the shape
    const int it = (int)(r / (uint32_t)sh.T);
    s.lt = (int)r - it * sh.T;
    s.T = sh.T;
    s.Tp = sh.Tp;
    s.item = pl.items[lo] + it;
    s.hk = it / sh.blocks_q;
    s.q0 = (it - s.hk * sh.blocks_q) * sh.per_q;
    s.Nq = min(sh.per_q, sh.total_q - s.q0);
    s.cnt = (int)min((long long)(s.T - s.lt), t_end - t);
}

// First tile of block c: the first one before which at least c / blocks of the cost lies.
template <int QB>
__device__ __forceinline__ long long first_tile(const Plan& pl, const Params& p, int c) {
    const long long total = pl.cost[p.B];
    if (c >= pl.blocks) return pl.tiles[p.B];
    const long long xc = total * c + pl.blocks - 1;           // (a 64-bit division takes a thousand cycles)
    const long long x = (unsigned long long)xc >> 32 ? xc / pl.blocks : (long long)((uint32_t)xc / (uint32_t)pl.blocks);
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pl.cost[mid] <= x) lo = mid; else hi = mid;
    }
    const Shape sh = shape_of<QB>(pl.len[lo], pl.nodes[lo], p.G);
    if (sh.T == 0) return pl.tiles[p.B];
    const int w = tile_cost(sh.per_q);
    const long long ci = (long long)sh.T * w + kItemCost, off = x - pl.cost[lo];
    const long long it = (unsigned long long)off >> 32 || ci >> 32 ? off / ci : (long long)((uint32_t)off / (uint32_t)ci);
    const long long rem = off - it * ci;                      // below T * w + the item's cost, T below 2^23
    const int lt = (int)(((uint32_t)rem + (uint32_t)w - 1u) / (uint32_t)w);
    return pl.tiles[lo] + it * sh.T + (lt < sh.T ? lt : sh.T);
}

template <int QB>
__device__ void make_plan(Plan& pl, const Params& p) {
    const int tid = threadIdx.x;
    for (int b = tid; b < p.B; b += kThreads) {
        const int L = min(max(p.seq_lens[b], 0), p.pages * kPageRows);
        const int Nb = p.n_active ? min(max(p.n_active[b], 0), p.N) : p.N;
        pl.len[b] = L;
        pl.nodes[b] = Nb;
    }
    __syncthreads();
    if (tid < 32) {                               // one warp scans the sequences, eight per lane
        long long t[8], c[8], ts = 0, cs = 0;
        int it[8], is = 0;
        const int per = (p.B + 31) / 32, b0 = tid * per;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t[i] = ts; c[i] = cs; it[i] = is;
            if (i < per && b0 + i < p.B) {
                const Shape sh = shape_of<QB>(pl.len[b0 + i], pl.nodes[b0 + i], p.G);
                const long long n = (long long)p.Hkv * sh.blocks_q;
                ts += n * sh.T;
                cs += n * ((long long)sh.T * tile_cost(sh.per_q) + kItemCost);
                is += (int)n;
            }
        }
        long long tb = ts, cb = cs;
        int ib = is;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long tv = __shfl_up_sync(0xffffffffu, tb, o), cv = __shfl_up_sync(0xffffffffu, cb, o);
            const int iv = __shfl_up_sync(0xffffffffu, ib, o);
            if (tid >= o) { tb += tv; cb += cv; ib += iv; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < per && b0 + i < p.B) {
                pl.tiles[b0 + i] = tb - ts + t[i];
                pl.cost[b0 + i] = cb - cs + c[i];
                pl.items[b0 + i] = ib - is + it[i];
            }
        if (tid == 31) { pl.tiles[p.B] = tb; pl.cost[p.B] = cb; pl.items[p.B] = ib; }
        __syncwarp();
        const long long all = __shfl_sync(0xffffffffu, tb, 31);
        if (tid == 0) pl.blocks = (int)min((long long)gridDim.x, all);
    }
    __syncthreads();
    if (tid <= (int)gridDim.x) pl.first[tid] = first_tile<QB>(pl, p, tid);
    __syncthreads();
}

template <int QB>
struct Small {
    unsigned long long full[kStages<QB>], empty[kStages<QB>];
    unsigned long long k_full[2], s_full[2], s_free[2], v_full[2], p_full[2], pv_done[2], q_full[2], piece_done[2], scales_full[8];
    unsigned long long drain;
    uint32_t tmem_base;
    int abort_flag;
    struct Merge {                                    // a cut work item, first or last of this block
        int before, cnt, T, hk, b, q0, Nq;            // tiles finished before this block's cnt, of T
        int block0;                                   // the block that has the item's first tile
        long long first;                              // the item's first tile
    } merge[2];
    int q_max;                                        // largest |query| of the first piece, as bits
    float q_factor[2];                                // brings sums over codes to score units
    int q_split[2];                                   // 1: the e4m3 parts are used, 0: the bf16 form
    int fmt[8];                                       // 1: the tile's values and weights are fp16, 0: bf16
    alignas(16) int row[2][QB];                                   // rows of q and out of the piece's columns
    alignas(16) float2 kab[4][kTile];                 // scale and offset of a tile's key rows, in score units
    alignas(16) unsigned short vab[8][2][kTile];      // scales and offsets of a tile's value rows, in the tile's format
    alignas(16) float q_sum[2][QB];
    alignas(16) float nref[2][QB];                    // running references of the two groups, negated
    alignas(16) float alpha[2][QB];                   // rescale factors of the two groups; at the end of a piece their weights
    alignas(16) float red[2][4][QB];
    alignas(16) uint64_t anc[MCSD_MAX_NODES * MCSD_MAX_WORDS];
    alignas(128) unsigned short ones[2][256];         // B operand of the row sums: bf16, fp16
    Piece piece[2];                                   // of the queries in the two buffers
    Plan plan;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, void* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void bulk_load_once(uint32_t dst, const void* src, uint32_t bytes, void* bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy) : "memory");
}
// (from the 16-byte boundary at or below src: values of the tree may start anywhere)
__device__ __forceinline__ void prefetch_l2(const void* src, uint32_t bytes) {
    src = reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(src) & ~(uintptr_t)15);
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy16_async(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
// One lane of a converged warp, the same one every time: it issues the MMAs and the commits that track them.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(r));
    return r != 0;
}
// tcgen05.mma by the calling lane, A operand in tensor memory or in shared memory
__device__ __forceinline__ void mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_sa(uint32_t d_tmem, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit(void* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// sixteen consecutive columns of this thread's lane
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void mma_ta8(uint32_t d_tmem, uint32_t a_tmem, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
// two numbers to e4m3 (b in the upper byte) and back
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
    unsigned short d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(b), "f"(a));
    return d;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t v) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)v));
    const __half2 x = *reinterpret_cast<const __half2*>(&h);
    return __half22float2(x);
}
// the largest and the smallest of three
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float d;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// (x & mask) | base, as the one instruction it is (left to itself the compiler makes it two)
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t base) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(x), "r"(mask), "r"(base));
    return d;
}
// codes (2i, 2i + 1) of a word as two numbers 16 + code: bf16 (code in mantissa bits 3..6) or fp16 (bits 6..9)
template <bool HALF>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i) {
    if (HALF) {
        const uint32_t x = i < 2 ? w << (6 - 4 * i) : w >> (4 * i - 6);
        return and_or(x, 0x03C003C0u, 0x4C004C00u);
    }
    const uint32_t x = i == 0 ? w << 3 : w >> (4 * i - 3);
    return and_or(x, 0x00780078u, 0x41804180u);
}
template <bool HALF>
__device__ __forceinline__ uint32_t fma_x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    if (HALF) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// eight weights as four pairs
template <bool HALF>
__device__ __forceinline__ uint4 pack8(const float (&y)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (HALF) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(y[2 * k + 1]), "f"(y[2 * k]));
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(y[2 * k + 1]), "f"(y[2 * k]));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// A key row's codes (its 16-byte pieces lie a page's rows apart) as bf16 numbers 16 + code in 64 columns of this thread's lane.
// (Rarely used, and kept out of the tile loop.)
__device__ __noinline__ void keys_to_bf16(const uint4* piece, uint32_t taddr) {
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
        const uint4 x = piece[c * kPageRows];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t y[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = code_pair<false>(w[e >> 2], e & 3);
        tc_st16(taddr + 16 * c, y);
    }
}
// Turns fp16 values into bf16 where they lie: 64 columns of this thread's lane.  (Rarely used, and kept out of the tile loop.)
__device__ __noinline__ void values_to_bf16(uint32_t taddr) {
    tc_fence_after();
#pragma unroll 1
    for (int c = 0; c < 8; ++c) {
        float y[8];
        tc_ld8(taddr + 8 * c, y);
        tc_wait_ld();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t w = __float_as_uint(y[k]);
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
            uint32_t b;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b) : "f"(v.y), "f"(v.x));
            y[k] = __uint_as_float(b);
        }
        tc_st8(taddr + 8 * c, y);
    }
    tc_wait_st();
}
// 32 x 32 bits, a row per lane: exchanges rows and columns
__device__ __forceinline__ uint32_t transpose_bits(uint32_t x, int lane) {
    uint32_t m = 0x0000FFFFu;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
        const uint32_t y = __shfl_xor_sync(0xffffffffu, x, s);
        x = lane & s ? (x & ~m) | ((y >> s) & m) : (x & m) | ((y & m) << s);
        m ^= m << (s >> 1);
    }
    return x;
}
// barrier over all softmax warps
__device__ __forceinline__ bool soft_sync_any(bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.or.pred q, 7, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r) : "r"((uint32_t)pred), "n"(kSoftThreads) : "memory");
    return r != 0;
}
// A row of values may be fp16: no value can leave its range, and neither scale nor values are so small that fp16's fixed
// spacing below 2^-14 would round them more coarsely than bf16 does.  False for scales that are not finite.
__device__ __forceinline__ bool fits_half(float scale, float offset) {
    const float o = fabsf(offset);
    return 31.f * scale + o <= 32768.f && (scale >= 6.103515625e-5f || (scale == 0.f && (o == 0.f || o >= 6.103515625e-5f)));
}

// Queries of a piece, sixteen lanes per row, lane c channels 8c .. 8c + 7.  In two steps, since the second needs the largest
// of them all.  Operand layouts: rows of 128 bytes with the 16-byte pieces of a row exchanged by row % 8; bf16 in two
// slabs of 64 channels, the e4m3 parts (high, low) behind them.  Codes come out of a word in the order 0 4 1 5 2 6 3 7, so the
// e4m3 channels are stored in that order.  Rows from the last query on are zeros.  Stacked query j of a key/value head
// is head j % G of its group, node j / G.
__device__ __forceinline__ int query_row(const Params& p, const Piece& s, int r) {   // row of q and out; below 65535 * 192
    const int j = s.q0 + r, n = j / p.G, h = s.hk * p.G + (j - n * p.G);
    return (s.b * p.Hkv * p.G + h) * p.N + n;
}
template <int QB>
__device__ __forceinline__ unsigned char* query_piece(unsigned char* q_buf, uint32_t buf, int r, int c) {   // of the bf16 form
    return q_buf + buf * (QB * 512) + (c >> 3) * (QB * 128) + r * 128 + (((c & 7) ^ (r & 7)) * 16);
}
// The row's sum, kept; returns the largest magnitude of the lane's channels.
template <int QB>
__device__ __forceinline__ float sum_query(Small<QB>* sm, uint32_t buf, int r, int c, uint4 v) {
    float2 sum = make_float2(0.f, 0.f);
    float top = 0.f;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        sum = add_f32x2(sum, x);
        top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
    }
    float all = sum.x + sum.y;
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) all += __shfl_xor_sync(0xffffffffu, all, x);
    if (c == 0) sm->q_sum[buf][r] = all;
    return top;
}
template <int QB>
__device__ __forceinline__ float load_query(Small<QB>* sm, unsigned char* q_buf, const Params& p, const Piece& s, uint32_t buf, int r, int c) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < s.Nq) {
        const int row = query_row(p, s, r);
        v = *reinterpret_cast<const uint4*>(p.q + (size_t)row * kD + c * 8);
        if (c == 0) sm->row[buf][r] = row;
    }
    *reinterpret_cast<uint4*>(query_piece<QB>(q_buf, buf, r, c)) = v;
    return sum_query<QB>(sm, buf, r, c, v);
}
// the power of two that brings the largest query to 128 .. 256 (e4m3 ends at 448)
__device__ __forceinline__ float query_scale(float top) {
    const int e = (int)(__float_as_uint(top) >> 23);               // of a number that is not negative
    return top > 0.f ? __uint_as_float((uint32_t)(min(max(127 + 7 - (e - 127), 10), 254)) << 23) : 1.f;
}
constexpr float kLeastTop = 16.f;                                  // of a row, next to the item's 128 .. 256
constexpr float kMostTop = 0x1p120f;                               // of an item, so that the power of two and its inverse are finite
// Returns 0 if the row's largest element is too far below the item's.
template <int QB>
__device__ __forceinline__ uint32_t split_query(unsigned char* q_buf, uint32_t buf, float scale, int r, int c) {
    const uint4 v = *reinterpret_cast<const uint4*>(query_piece<QB>(q_buf, buf, r, c));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16) * scale;
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u) * scale;
    }
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {                                    // channels 0 4 1 5, then 2 6 3 7
        const float a = x[2 * i], b = x[2 * i + 4], d = x[2 * i + 1], e = x[2 * i + 5];
        const uint32_t h0 = to_e4m3x2(a, b), h1 = to_e4m3x2(d, e);
        const float2 f0 = from_e4m3x2(h0), f1 = from_e4m3x2(h1);
        hi[i] = h0 | (h1 << 16);
        lo[i] = to_e4m3x2(a - f0.x, b - f0.y) | (to_e4m3x2(d - f1.x, e - f1.y) << 16);
    }
    unsigned char* at = q_buf + buf * (QB * 512) + QB * 256 + r * 128 + (((c >> 1) ^ (r & 7)) * 16) + (c & 1) * 8;
    *reinterpret_cast<uint2*>(at) = make_uint2(hi[0], hi[1]);
    *reinterpret_cast<uint2*>(at + QB * 128) = make_uint2(lo[0], lo[1]);
    const float top = max3(max3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2])), max3(fabsf(x[3]), fabsf(x[4]), fabsf(x[5])), fmaxf(fabsf(x[6]), fabsf(x[7])));
    return __ballot_sync(0xffffffffu, top >= kLeastTop) & (0xFFFFu << (threadIdx.x & 16u));
}
// the largest finite magnitude of the lane's channels of rows r, r + step, ... (rarely used)
template <int QB>
__device__ __noinline__ float finite_top(unsigned char* q_buf, uint32_t buf, int r, int rows, int step, int c) {
    uint32_t top = 0;
#pragma unroll 1
    for (; r < rows; r += step) {
        const uint4 v = *reinterpret_cast<const uint4*>(query_piece<QB>(q_buf, buf, r, c));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = (w[i] << 16) & 0x7FFF0000u, b = w[i] & 0x7FFF0000u;
            top = max(top, max(a < 0x7F800000u ? a : 0u, b < 0x7F800000u ? b : 0u));
        }
    }
    return __uint_as_float(top);
}

template <int QB>
__global__ void __launch_bounds__(kThreads, 1)
tree_attention_kv4_kernel(const Params p) {
    using Col = Columns<QB>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);   // (an offset: the compiler keeps knowing it is shared memory)
    unsigned char* q_buf = smem;                      // two buffers of QB rows: [2 bf16 slabs, high, low][QB rows][128 bytes]
    unsigned char* p_buf = q_buf + 2 * QB * 512;      // P^T of the two groups: [QB / 8][128 keys][16 bytes]
    unsigned char* ring = p_buf + 2 * QB * 256;
    Small<QB>* sm = reinterpret_cast<Small<QB>*>(ring + kStages<QB> * kStageBytes);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- set-up; what comes before the wait touches no global memory and overlaps the tail of the preceding kernel
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < kStages<QB>; ++i) { mbar_init(&sm->full[i], 1); mbar_init(&sm->empty[i], 8); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm->k_full[i], 4);
            mbar_init(&sm->s_full[i], 1);
            mbar_init(&sm->s_free[i], 4);
            mbar_init(&sm->v_full[i], 4);
            mbar_init(&sm->p_full[i], 4);
            mbar_init(&sm->pv_done[i], 1);
            mbar_init(&sm->q_full[i], 1);
            mbar_init(&sm->piece_done[i], kSoftThreads / 32);
        }
        for (int i = 0; i < 8; ++i) mbar_init(&sm->scales_full[i], 4);
        mbar_init(&sm->drain, 2);
        sm->abort_flag = 0;
        sm->q_max = 0;
        sm->q_split[0] = 1;
        sm->merge[0].T = sm->merge[1].T = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 256) { sm->ones[0][tid] = 0x3F80; sm->ones[1][tid] = 0x3C00; }
    fence_async_smem();                               // read by the tensor cores through the async proxy
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = tid - kMaxBatchTc; i >= 0 && i < p.N * p.words; i += kThreads - kMaxBatchTc) sm->anc[i] = p.anc[i];
    make_plan<QB>(sm->plan, p);
    const Plan& pl = sm->plan;
    const long long t_begin = pl.first[blockIdx.x], t_end = pl.first[blockIdx.x + 1];
    if (t_begin >= t_end) return;                     // uniform for the whole block: nothing allocated yet

    WorkspaceHeader* const hdr = p.header;
    int* const abort_flag = &sm->abort_flag;
    uint32_t tmem = 0;
    if (warp != kCopyWarp) {                          // whose first loads are on their way meanwhile
        if (warp == kScoreWarp) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem_base)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        // the first piece's queries, by everybody
        Piece s;
        piece_at<QB>(pl, p, t_begin, t_end, s);
        const int r0 = warp > kCopyWarp ? (tid >> 4) - 2 : tid >> 4, c = tid & 15, rows = (s.Nq + 15) & ~15;
        constexpr int at_once = (kThreads - 32) / 16;
        float top = 0.f;
        for (int r = r0; r < rows; r += at_once) top = fmaxf(top, load_query<QB>(sm, q_buf, p, s, 0, r, c));
        top = warp_max_f32(top);
        if (lane == 0) atomicMax(&sm->q_max, __float_as_int(top));
        tc_fence_before();
        asm volatile("bar.sync 9, %0;" ::"n"(kThreads - 32) : "memory");
        tc_fence_after();
        tmem = *(volatile uint32_t*)&sm->tmem_base;
        top = __int_as_float(sm->q_max);
        if (!(top < INFINITY)) {                      // an infinite element says nothing about the others
            asm volatile("bar.sync 9, %0;" ::"n"(kThreads - 32) : "memory");
            if (tid == 0) sm->q_max = 0;
            asm volatile("bar.sync 9, %0;" ::"n"(kThreads - 32) : "memory");
            top = warp_max_f32(finite_top<QB>(q_buf, 0, r0, rows, at_once, c));
            if (lane == 0) atomicMax(&sm->q_max, __float_as_int(top));
            asm volatile("bar.sync 9, %0;" ::"n"(kThreads - 32) : "memory");
            top = __int_as_float(sm->q_max);
        }
        const float scale = query_scale(top);
        bool fine = top < kMostTop;
        for (int r = r0; r < rows; r += at_once) fine &= split_query<QB>(q_buf, 0, scale, r, c) != 0u || r >= s.Nq || top == 0.f;
        if (!fine) sm->q_split[0] = 0;
        if (tid == 0) { sm->q_factor[0] = 512.f / scale; sm->piece[0] = s; }
        fence_async_smem();
        asm volatile("bar.sync 9, %0;" ::"n"(kThreads - 32) : "memory");
        if (!sm->q_split[0]) sm->q_factor[0] = 1.f;   // (by every thread that reads it)
    }

    // Tiles of this block are numbered g = 0, 1, ... across its pieces; f counts those that come through the ring.
    if (warp == kCopyWarp) {
        if (lane == 0) {
            const bool once = (long long)p.G * p.N <= QB;       // one query block: no other work item reads the pages
            const uint64_t pol = l2_policy_evict_first();
            uint32_t f = 0;
            bool ok = true;
            for (long long t = t_begin; t < t_end && ok;) {
                Piece s;
                piece_at<QB>(pl, p, t, t_end, s);
                const unsigned char* head = p.cache + ((size_t)s.b * p.Hkv + s.hk) * p.pages * kPageBytes;
                if (s.lt + s.cnt > s.Tp && s.Nb > 0) {              // the rows of the tree, into L2 long before they are read
                    const size_t row = ((size_t)s.b * p.Hkv + s.hk) * p.N * kD;
                    prefetch_l2(p.k_tree + row, (uint32_t)s.Nb * kD * 2);
                    prefetch_l2(p.v_tree + row, (uint32_t)s.Nb * kD * 2);
                }
                for (int i = s.lt; i < min(s.lt + s.cnt, s.Tp) && ok; ++i, ++f) {
                    const uint32_t st = f % kStages<QB>;
                    if (f >= kStages<QB>) ok = mbar_wait(&sm->empty[st], (f / kStages<QB> - 1u) & 1u, abort_flag, hdr, 31);
                    if (!ok) break;
                    const uint32_t bytes = (uint32_t)(min(kTile, s.L - i * kTile) + kPageRows - 1) / kPageRows * kPageBytes;
                    mbar_expect_tx(&sm->full[st], bytes);
                    const uint32_t dst = smem_u32(ring) + st * kStageBytes;
                    const unsigned char* src = head + (size_t)i * kStageBytes;
                    if (once) bulk_load_once(dst, src, bytes, &sm->full[st], pol);
                    else bulk_load(dst, src, bytes, &sm->full[st]);
                }
                t += s.cnt;
            }
            if (!ok) {                                // gave up: let the copies already issued land before the block exits
                for (uint32_t x = f > kStages<QB> ? f - kStages<QB> : 0; x < f; ++x) {
                    const long long t0 = clock64();
                    while (!mbar_try_wait(&sm->full[x % kStages<QB>], (x / kStages<QB>) & 1u) && clock64() - t0 < kSpinCycles / 8) {}
                }
            }
        }
    } else if (warp == kScoreWarp) {
        const uint64_t dq0 = smem_desc(smem_u32(q_buf), 16, 1024, 2);
        constexpr uint32_t q_slab = (QB * 128) >> 4, q_next = (QB * 512) >> 4;
        uint32_t g = 0, seg = 0;
        bool ok = true;
        for (long long t = t_begin; t < t_end && ok; ++seg) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            ok = mbar_wait(&sm->q_full[seg & 1u], (seg >> 1) & 1u, abort_flag, hdr, 32);
            const uint32_t idesc = instr_desc((s.Nq + 15) & ~15, 0, 0), idesc8 = idesc & ~((1u << 7) | (1u << 10));   // e4m3 is format 0
            const uint64_t dq = dq0 + (seg & 1u) * q_next;
            const int narrow = sm->q_split[seg & 1u] ? s.Tp : 0;
            for (int i = s.lt; i < s.lt + s.cnt && ok; ++i, ++g) {
                const uint32_t buf = g & 1u;
                ok = mbar_wait(&sm->k_full[buf], (g >> 1) & 1u, abort_flag, hdr, 33);
                if (ok && g >= 2) ok = mbar_wait(&sm->s_free[buf], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 46);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t d = tmem + Col::S + buf * QB;
                    if (i < narrow) {                 // 32 channels per MMA: high parts, then low parts
                        const uint32_t ka = tmem + Col::K + buf * 32;
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            mma_ta8(d, ka + 8 * (k & 3), dq + (uint32_t)(2 + (k >> 2)) * q_slab + (uint32_t)(k & 3) * 2u, idesc8, k > 0);
                    } else {
#pragma unroll 1
                        for (int k = 0; k < 8; ++k)
                            mma_ta(d, tmem + Col::K + 8 * k, dq + (uint32_t)(k >> 2) * q_slab + (uint32_t)(k & 3) * 2u, idesc, k > 0);
                    }
                    commit(&sm->s_full[buf]);
                }
                __syncwarp();
            }
            t += s.cnt;
        }
        if (elect_one()) commit(&sm->drain);          // all MMAs have finished before tensor memory is released
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&sm->drain, 0) && clock64() - t0 < kSpinCycles) {}
    } else if (warp == kProductWarp) {
        const uint64_t dp0 = smem_desc(smem_u32(p_buf), 128, 2048, 0);
        const uint64_t d1 = smem_desc(smem_u32(sm->ones), 128, 256, 0);
        constexpr uint32_t p_next = (QB * 256) >> 4, one_next = 512 >> 4;
        const uint32_t idesc_lb = instr_desc(16, 1, 0);
        uint32_t g = 0;
        bool ok = true;
        for (long long t = t_begin; t < t_end && ok;) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            const uint32_t idesc_b = instr_desc((s.Nq + 15) & ~15, 0, 1);
            for (int i = 0; i < s.cnt; ++i, ++g) {
                const uint32_t hb = g & 1u;
                ok = mbar_wait(&sm->v_full[hb], (g >> 1) & 1u, abort_flag, hdr, 34);
                if (ok) ok = mbar_wait(&sm->p_full[hb], (g >> 1) & 1u, abort_flag, hdr, 35);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    // fp16 operands are format 0 of both operand fields, bf16 is 1
                    const uint32_t half = sm->fmt[g & 7u];
                    const uint32_t fp16 = ~(half ? (1u << 7) | (1u << 10) : 0u), idesc = idesc_b & fp16, idesc_l = idesc_lb & fp16;
                    const uint32_t d = tmem + Col::O + hb * QB, l = tmem + Col::L + hb * 16, va = tmem + Col::V + hb * 64;
                    const uint64_t dp = dp0 + hb * p_next, d1h = d1 + half * one_next;
                    const uint32_t more = i >= 2;     // a group's first tile of a piece overwrites
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        mma_ta(d, va + 8 * k, dp + (uint32_t)(k * (256 >> 4)), idesc, more | (uint32_t)(k > 0));
                        // (P^T read as the A operand, queries on the lanes; lanes past the last query hold nothing of use)
                        mma_sa(l, dp + (uint32_t)(k * (256 >> 4)), d1h, idesc_l, more | (uint32_t)(k > 0));
                    }
                    commit(&sm->pv_done[hb]);
                }
                __syncwarp();
            }
            t += s.cnt;
        }
        if (elect_one()) commit(&sm->drain);
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&sm->drain, 0) && clock64() - t0 < kSpinCycles) {}
    } else if (warp == kQueryWarp) {
        // queries of the next piece (the first one's are there), two rows at a time; and, a while after a piece of a cut item is
        // done, the count of the item's tiles (who brings the last ones merges, see the end of the kernel)
        const int sub = lane >> 4, c = lane & 15;
        uint32_t seg = 0;
        bool ok = true;
        auto finish = [&](uint32_t done) {                    // piece number `done`, the last or the one before
            ok = mbar_wait(&sm->piece_done[done & 1u], (done >> 1) & 1u, abort_flag, hdr, 36);
            const Piece& s = sm->piece[done & 1u];
            if (ok && lane == 0 && s.cnt != s.T) {
                auto& m = sm->merge[done > 0 ? 1 : 0];
                m.b = s.b; m.hk = s.hk; m.q0 = s.q0; m.Nq = s.Nq; m.T = s.T; m.cnt = s.cnt;
                m.first = pl.tiles[s.b] + (long long)(s.item - pl.items[s.b]) * s.T;
                int lo = blockIdx.x;
                if (s.lt > 0) {                               // the last block that does not start behind the item's first tile
                    lo = 0;
                    for (int hi = blockIdx.x; hi - lo > 1;) {
                        const int mid = (lo + hi) >> 1;
                        if (pl.first[mid] <= m.first) lo = mid; else hi = mid;
                    }
                }
                m.block0 = lo;
                int* const counter = p.counters + lo * kCountersPerBlock;
                __threadfence();
                m.before = atomicAdd(counter, s.cnt);
                if (m.before + s.cnt == s.T) *counter = 0;
            }
            __syncwarp();
        };
        for (long long t = t_begin; t < t_end && ok; ++seg) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            const uint32_t buf = seg & 1u;
            if (seg > 0) {
                if (seg >= 2) finish(seg - 2u);
                if (!ok) break;
                const int rows = (s.Nq + 15) & ~15;
                for (int r = lane; r < s.Nq; r += 32) sm->row[buf][r] = query_row(p, s, r);
                __syncwarp();
                // all rows are on their way at once: a short work item has little time to hide this behind
                for (int r = sub; r < rows; r += 2) {
                    unsigned char* const to = query_piece<QB>(q_buf, buf, r, c);
                    if (r < s.Nq) copy16_async(to, p.q + (size_t)(uint32_t)sm->row[buf][r] * kD + c * 8);
                    else *reinterpret_cast<uint4*>(to) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("cp.async.wait_all;" ::: "memory");       // (a lane reads below what it has copied itself)
                float top = 0.f;
#pragma unroll 4
                for (int r = sub; r < rows; r += 2)
                    top = fmaxf(top, sum_query<QB>(sm, buf, r, c, *reinterpret_cast<const uint4*>(query_piece<QB>(q_buf, buf, r, c))));
                top = warp_max_f32(top);
                if (!(top < INFINITY)) {
                    top = warp_max_f32(finite_top<QB>(q_buf, buf, sub, rows, 2, c));
                }
                const float scale = query_scale(top);
                bool fine = top < kMostTop;
#pragma unroll 2
                for (int r = sub; r < rows; r += 2) fine &= split_query<QB>(q_buf, buf, scale, r, c) != 0u || r >= s.Nq || top == 0.f;
                fine = __all_sync(0xffffffffu, fine);
                if (lane == 0) {
                    sm->q_factor[buf] = fine ? 512.f / scale : 1.f;
                    sm->q_split[buf] = fine;
                    sm->piece[buf] = s;
                }
                fence_async_smem();
                __syncwarp();
            }
            if (lane == 0) mbar_arrive(&sm->q_full[buf]);
            t += s.cnt;
        }
        if (ok && seg >= 2) finish(seg - 2u);
        if (ok) finish(seg - 1u);
    } else if (warp < kValueWarp) {
        // ---- keys: thread r owns key row r of a tile
        const int r = tid;
        const uint32_t lane_addr = tmem + ((uint32_t)(warp * 32) << 16);
        uint32_t g = 0, f = 0, seg = 0;
        bool bad = false, gone = false, wide = false;         // wide: the previous tile took both buffers
        for (long long t = t_begin; t < t_end && !gone; ++seg) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            // (the first piece's queries are there since the set-up)
            if (seg > 0) bad |= !mbar_wait(&sm->q_full[seg & 1u], (seg >> 1) & 1u, abort_flag, hdr, 51);
            const int narrow = sm->q_split[seg & 1u] ? s.Tp : 0;   // tiles from here on take both buffers
            for (int i = s.lt; i < s.lt + s.cnt; ++i, ++g) {
                const uint32_t buf = g & 1u;
                const uint32_t st = f % kStages<QB>;
                if (i < s.Tp) bad |= !mbar_wait(&sm->full[st], (f / kStages<QB>) & 1u, abort_flag, hdr, 37);
                // Scales of the tile's value rows, thread r the row r, rounded to fp16.  Rows past the end of the prefix have
                // probability zero but may hold anything, and 0 * NaN would be NaN: their scale and offset are zero.
                const unsigned char* page = ring + st * kStageBytes + warp * kPageBytes;   // rows 32 warp .. of the tile
                const unsigned short* sc = reinterpret_cast<const unsigned short*>(page + kv4_scales_at(kD)) + lane;
                uint32_t a16 = 0, b16 = 0;
                if (i < s.Tp && r < s.L - i * kTile) { a16 = sc[2 * kPageRows]; b16 = sc[3 * kPageRows]; }
                const float va = bf16_bits_to_f32(a16), vb = bf16_bits_to_f32(b16);
                const bool odd = group_sync_any(8, bad || i >= s.Tp || !fits_half(va, vb));   // not fp16
                if (odd) {
                    gone = group_sync_any(8, bad);
                    if (gone) break;
                }
                // (The entry of tile g - 8.  The scores of tile g - 3 are done; so softmax had stored the weights of tile g - 5, for which it
                // waited for the products of tile g - 7, and those of tile g - 8 came before.)
                sm->vab[g & 7u][0][r] = odd ? (unsigned short)a16 : __half_as_ushort(__float2half_rn(va));
                sm->vab[g & 7u][1][r] = odd ? (unsigned short)b16 : __half_as_ushort(__float2half_rn(vb));
                if (r == 0) sm->fmt[g & 7u] = !odd;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->scales_full[g & 7u]);
                // A buffer is free once the scores of the tile that used it are done: the tile before last, and the last one
                // too where either of the two takes both buffers.  They were issued after the softmax warps had taken
                // the scores and the scales of tile g - 4, whose entry is rewritten below.
                if (g >= 2) bad |= !mbar_wait(&sm->s_full[buf], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 38);
                if (g >= 1 && (wide || i >= narrow)) bad |= !mbar_wait(&sm->s_full[buf ^ 1u], ((g - 1u) >> 1) & 1u, abort_flag, hdr, 47);
                tc_fence_after();
                wide = i >= narrow;
                if (i < narrow) {
                    const uint4* piece = reinterpret_cast<const uint4*>(page) + lane;
                    const float a = bf16_bits_to_f32(sc[0]), b = bf16_bits_to_f32(sc[kPageRows]);
                    sm->kab[g & 3u][r] = make_float2(a * p.scale_log2, fmaf(16.f, a, b) * p.scale_log2);
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        const uint4 x0 = piece[2 * c * kPageRows], x1 = piece[(2 * c + 1) * kPageRows];
                        const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
                        uint32_t y[16];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            y[2 * e] = w[e] & 0x0F0F0F0Fu;
                            y[2 * e + 1] = (w[e] >> 4) & 0x0F0F0F0Fu;
                        }
                        tc_st16(lane_addr + Col::K + buf * 32 + 16 * c, y);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->empty[st]);
                    ++f;
                } else if (i < s.Tp) {
                    sm->kab[g & 3u][r] = make_float2(bf16_bits_to_f32(sc[0]) * p.scale_log2, bf16_bits_to_f32(sc[kPageRows]) * p.scale_log2);
                    keys_to_bf16(reinterpret_cast<const uint4*>(page) + lane, lane_addr + Col::K);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->empty[st]);
                    ++f;
                } else {
                    const int n = (i - s.Tp) * kTile + r;
                    sm->kab[g & 3u][r] = make_float2(p.scale_log2, 0.f);
                    const uint4* row = reinterpret_cast<const uint4*>(p.k_tree + (((size_t)s.b * p.Hkv + s.hk) * p.N + n) * kD);
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t y[16];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint4 v = n < s.Nb ? row[4 * c + e] : make_uint4(0, 0, 0, 0);
                            y[4 * e] = v.x; y[4 * e + 1] = v.y; y[4 * e + 2] = v.z; y[4 * e + 3] = v.w;
                        }
                        tc_st16(lane_addr + Col::K + 16 * c, y);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->k_full[buf]);
            }
            t += s.cnt;
        }
    } else if (warp < kSoftWarp) {
        // ---- values: thread d owns channel d
        const int d = tid & 127;
        const uint32_t vg = (uint32_t)(warp - kValueWarp) >> 2;   // takes the tiles with g % 2 == vg
        const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + Col::V;
        uint32_t g = 0, f = 0;
        bool ok = true;
        for (long long t = t_begin; t < t_end && ok;) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            for (int i = s.lt; i < s.lt + s.cnt; ++i, ++g) {
                if ((g & 1u) != vg) {
                    if (i < s.Tp) ++f;
                    continue;
                }
                const uint32_t dst = lane_addr + (g & 1u) * 64;
                const uint32_t st = f % kStages<QB>;
                // (the key warps have seen the tile arrive before they announce its scales)
                ok = mbar_wait(&sm->scales_full[g & 7u], (g >> 3) & 1u, abort_flag, hdr, 39);
                // the buffer is free once the products of the tile that used it are done
                if (ok && g >= 2) ok = mbar_wait(&sm->pv_done[vg], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 40);
                if (!ok) break;
                tc_fence_after();
                if (i < s.Tp) {
                    if (!mbar_try_wait(&sm->full[st], (f / kStages<QB>) & 1u)) {                  // (has completed)
                        *(volatile int*)abort_flag = 1;
                        hdr->detail = 52;
                        hdr->status = MCSD_ERR_TIMEOUT;
                        ok = false;
                        break;
                    }
                    const bool half = sm->fmt[g & 7u];
                    const unsigned char* codes = ring + st * kStageBytes + kv4_values_at(kD) + d * 16;
                    const uint4* sa = reinterpret_cast<const uint4*>(sm->vab[g & 7u][0]);
                    const uint4* sb = reinterpret_cast<const uint4*>(sm->vab[g & 7u][1]);
                    auto unpack = [&](auto half_tag) {
                        constexpr bool HALF = decltype(half_tag)::value;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            const uint4 x = *reinterpret_cast<const uint4*>(codes + c * kPageBytes);
                            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                            uint32_t y[16];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint4 a = sa[4 * c + j], b = sb[4 * c + j];
                                y[4 * j] = fma_x2<HALF>(code_pair<HALF>(w[j], 0), a.x, b.x);
                                y[4 * j + 1] = fma_x2<HALF>(code_pair<HALF>(w[j], 1), a.y, b.y);
                                y[4 * j + 2] = fma_x2<HALF>(code_pair<HALF>(w[j], 2), a.z, b.z);
                                y[4 * j + 3] = fma_x2<HALF>(code_pair<HALF>(w[j], 3), a.w, b.w);
                            }
                            tc_st16(dst + 16 * c, y);
                        }
                    };
                    if (half) unpack(std::true_type{}); else unpack(std::false_type{});
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->empty[st]);
                    ++f;
                } else {
                    const int n0 = (i - s.Tp) * kTile, n1 = min(kTile, s.Nb - n0);
                    const unsigned short* col = reinterpret_cast<const unsigned short*>(p.v_tree) + (((size_t)s.b * p.Hkv + s.hk) * p.N + n0) * kD + d;
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t y[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int n = 32 * c + 2 * e;
                            const uint32_t lo = n < n1 ? col[(size_t)n * kD] : 0u, hi = n + 1 < n1 ? col[(size_t)(n + 1) * kD] : 0u;
                            y[e] = lo | (hi << 16);
                        }
                        tc_st16(dst + 16 * c, y);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->v_full[g & 1u]);
            }
            t += s.cnt;
        }
    } else {
        // ---- softmax, epilogue: group wg has the tiles with g % 2 == wg, thread r key row r
        const int wg = (warp - kSoftWarp) >> 2, wq = warp & 3, r = tid & 127, bar_id = 1 + wg;
        const uint32_t lane_addr = tmem + ((uint32_t)(wq * 32) << 16);
        const uint32_t s_addr = lane_addr + Col::S + wg * QB;
        unsigned char* const p_own = p_buf + wg * (QB * 256) + r * 16;
        float* const nref = sm->nref[wg];
        float* const alph = sm->alpha[wg];
        uint32_t g_piece = 0, seg = 0;                           // tiles of this block before the piece
        bool failed = false, gone = false;                       // gone: all threads know that one has failed
        for (long long t = t_begin; t < t_end; ++seg) {
            if (!mbar_wait(&sm->q_full[seg & 1u], (seg >> 1) & 1u, abort_flag, hdr, 48)) failed = true;
            const Piece s = sm->piece[seg & 1u];
            if (soft_sync_any(failed)) break;                    // (all leave or none)
            const int n8 = (s.Nq + 7) >> 3;
            const bool own_col = r < 8 * n8;                     // thread r keeps column r's reference
            const float* qs = sm->q_sum[seg & 1u];
            const uint32_t g_end = g_piece + (uint32_t)s.cnt;
            const uint32_t g_own = g_piece + ((g_piece ^ (uint32_t)wg) & 1u);   // the group's first tile, if below g_end
            bool deep = false;                                   // has met weights too small for fp16
            for (uint32_t g = g_own; g < g_end; g += 2) {
                const int i = s.lt + (int)(g - g_piece);
                const bool tree = i >= s.Tp;
                const int key = (tree ? i - s.Tp : i) * kTile + r;
                const bool plain = !tree && (i + 1) * kTile <= s.L;   // every key there and visible to every query
                unsigned long long cm = 0;                       // columns that see this thread's key
                if (!plain) {
                    if (!tree) {
                        if (key < s.L) cm = ~0ull;
                    } else {
                        const int key0 = (i - s.Tp) * kTile + wq * 32;   // the warp's first key
                        const uint32_t* const anc32 = reinterpret_cast<const uint32_t*>(sm->anc) + (key0 >> 5);
                        uint32_t m[2];
#pragma unroll
                        for (int x = 0; x < 2; ++x) {            // lane c: which of the warp's keys column 32 x + c sees
                            const int c = 32 * x + lane;
                            m[x] = c < s.Nq && key0 < s.Nb ? anc32[(s.q0 + c) / p.G * (2 * p.words)] : 0u;
                            m[x] = transpose_bits(m[x], lane);   // lane r: which of those columns see key r
                        }
                        cm = key < s.Nb ? m[0] | ((unsigned long long)m[1] << 32) : 0ull;
                    }
                }
                if (!mbar_wait(&sm->s_full[wg], (g >> 1) & 1u, abort_flag, hdr, 41)) failed = true;
                tc_fence_after();
                bool half = sm->fmt[g & 7u] && !deep;
                const bool first = g == g_own;
                float2 ab = sm->kab[g & 3u][r];
                if (!tree) ab.x *= sm->q_factor[seg & 1u];
                const float2 a2 = make_float2(ab.x, ab.x), b2 = make_float2(ab.y, ab.y);
                // The first references of a piece come from the largest of four keys' scores (one per warp).  Any reference gives
                // the same result as long as the weights keep their precision; one that is exceeded too far is raised
                // below, and weights that are too small for fp16 make the tile, and the rest of the piece, bf16.  A tile with
                // a mask takes exact column maxima instead.
                if (first && plain) {
#pragma unroll 1
                    for (int j = 0; j < n8; ++j) {
                        float y[8];
                        tc_ld8(s_addr + 8 * j, y);
                        const float4 q0 = *reinterpret_cast<const float4*>(qs + 8 * j), q1 = *reinterpret_cast<const float4*>(qs + 8 * j + 4);
                        tc_wait_ld();
                        if (lane == 0) {
                            float4* const to = reinterpret_cast<float4*>(&sm->red[wg][wq][8 * j]);
                            to[0] = make_float4(fmaf(y[0], ab.x, q0.x * ab.y), fmaf(y[1], ab.x, q0.y * ab.y), fmaf(y[2], ab.x, q0.z * ab.y), fmaf(y[3], ab.x, q0.w * ab.y));
                            to[1] = make_float4(fmaf(y[4], ab.x, q1.x * ab.y), fmaf(y[5], ab.x, q1.y * ab.y), fmaf(y[6], ab.x, q1.z * ab.y), fmaf(y[7], ab.x, q1.w * ab.y));
                        }
                    }
                    group_sync_any(bar_id, false);
                    if (own_col) {
                        const float top = fmaxf(fmaxf(sm->red[wg][0][r], sm->red[wg][1][r]), fmaxf(sm->red[wg][2][r], sm->red[wg][3][r]));
                        nref[r] = -fmaxf(top - kFirstLog, -1e30f);
                    }
                    group_sync_any(bar_id, false);
                }
                // Then an optimistic sweep; where a score exceeds its reference by more than 2^kTopLog, new references and the
                // same again; where weights are too small for fp16, the same again in bf16.  (Such weights are nothing
                // beside a key that outweighs them all, but all there is to the result where that key's value is zero.)
                bool raise = first && !plain, raised = false;
                for (;;) {
                    if (raise) {
                        raised = true;
#pragma unroll 1
                        for (int j = 0; j < n8; ++j) {
                            float y[8];
                            tc_ld8(s_addr + 8 * j, y);
                            tc_wait_ld();
                            float mine = -INFINITY;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float x = fmaf(y[k], ab.x, qs[8 * j + k] * ab.y);
                                const float mx = warp_max_f32((plain || ((cm >> (8 * j + k)) & 1ull)) ? x : -INFINITY);
                                if (lane == k) mine = mx;
                            }
                            if (lane < 8) sm->red[wg][wq][8 * j + lane] = mine;
                        }
                        group_sync_any(bar_id, false);
                        if (own_col) {
                            const float top = fmaxf(fmaxf(sm->red[wg][0][r], sm->red[wg][1][r]), fmaxf(sm->red[wg][2][r], sm->red[wg][3][r]));
                            // (a column that has seen no key yet keeps one below any score)
                            const float old = first ? -1e30f : -nref[r], now = fmaxf(old, top - kFirstLog);
                            nref[r] = -now;
                            alph[r] = exp2f(old - now);
                        }
                        group_sync_any(bar_id, false);
                        if (!first) {
                            // (the accumulators are current once the products of the group's previous tile are done)
                            if (!mbar_wait(&sm->pv_done[wg], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 42)) failed = true;
                            tc_fence_after();
#pragma unroll 1
                            for (int j = 0; j < n8; ++j) {
                                float o[8];
                                tc_ld8(lane_addr + Col::O + wg * QB + 8 * j, o);
                                tc_wait_ld();
#pragma unroll
                                for (int k = 0; k < 8; ++k) o[k] *= alph[8 * j + k];
                                tc_st8(lane_addr + Col::O + wg * QB + 8 * j, o);
                            }
                            const float l = tc_ld1(lane_addr + Col::L + wg * 16);   // of query r
                            tc_wait_ld();
                            tc_st1(lane_addr + Col::L + wg * 16, own_col ? l * alph[r] : l);
                            tc_wait_st();
                        }
                    }
                    // scores of this thread's key relative to the references, exponentiated, packed, stored
                    float dmax = -INFINITY, dmin = INFINITY;
                    // P^T may be written once the products of the group's previous tile are done (they are, nearly always)
                    auto p_free = [&]() {
                        if (g >= 2 && !mbar_wait(&sm->pv_done[wg], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 43)) failed = true;
                    };
                    auto scores = [&](float (&y)[8], float (&x)[8], int j) {
#pragma unroll
                        for (int k = 0; k < 8; k += 4) {
                            const float4 q = *reinterpret_cast<const float4*>(qs + 8 * j + k), m = *reinterpret_cast<const float4*>(nref + 8 * j + k);
                            const float2 u = fma_f32x2(make_float2(y[k], y[k + 1]), a2, fma_f32x2(make_float2(q.x, q.y), b2, make_float2(m.x, m.y)));
                            const float2 v = fma_f32x2(make_float2(y[k + 2], y[k + 3]), a2, fma_f32x2(make_float2(q.z, q.w), b2, make_float2(m.z, m.w)));
                            x[k] = u.x; x[k + 1] = u.y; x[k + 2] = v.x; x[k + 3] = v.y;
                        }
                    };
                    if (plain && half) {                         // nearly all tiles
                        // (the next column group is on its way as soon as this one is out of the load's registers)
                        float y[8];
                        tc_ld8(s_addr, y);
                        p_free();
#pragma unroll 1
                        for (int j = 0; j < n8; ++j) {
                            float x[8];
                            tc_wait_ld();
                            scores(y, x, j);
                            if (j + 1 < n8) tc_ld8(s_addr + 8 * j + 8, y);
#pragma unroll
                            for (int k = 0; k < 8; k += 2) {
                                dmax = max3(dmax, x[k], x[k + 1]);
                                dmin = min3(dmin, x[k], x[k + 1]);
                                x[k] = ex2_approx(x[k]);
                                x[k + 1] = ex2_approx(x[k + 1]);
                            }
                            *reinterpret_cast<uint4*>(p_own + j * 2048) = pack8<true>(x);
                        }
                    } else {                                     // masks, bf16
                        float y[8];
                        tc_ld8(s_addr, y);
                        p_free();
#pragma unroll 1
                        for (int j = 0; j < n8; ++j) {
                            const uint32_t bits = plain ? 0xFFu : (uint32_t)(cm >> (8 * j));
                            float x[8];
                            tc_wait_ld();
                            scores(y, x, j);
                            if (j + 1 < n8) tc_ld8(s_addr + 8 * j + 8, y);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const bool seen = (bits >> k) & 1u;
                                dmin = fminf(dmin, seen ? x[k] : INFINITY);
                                x[k] = seen ? x[k] : -INFINITY;
                                dmax = fmaxf(dmax, x[k]);
                                x[k] = ex2_approx(x[k]);
                            }
                            *reinterpret_cast<uint4*>(p_own + j * 2048) = half ? pack8<true>(x) : pack8<false>(x);
                        }
                    }
                    const bool over = dmax > kTopLog && !raised;
                    if (!group_sync_any(bar_id, over || (half && dmin < kLowLog) || failed)) break;   // one vote of the four warps
                    gone = group_sync_any(bar_id, failed);
                    if (gone) break;
                    raise = group_sync_any(bar_id, over);
                    if (!raise) {
                        deep = true;
                        half = false;
                    }
                }
                if (gone) break;
                if (deep && sm->fmt[g & 7u]) {
                    // the value warps have stored fp16 and wait for the products, the products wait for this group
                    if (!mbar_wait(&sm->v_full[wg], (g >> 1) & 1u, abort_flag, hdr, 50)) failed = true;
                    __syncwarp();
                    values_to_bf16(lane_addr + Col::V + wg * 64);
                    group_sync_any(bar_id, false);               // everybody in the group has read the format
                    if (r == 0) sm->fmt[g & 7u] = 0;
                }
                tc_fence_before();
                if (lane == 0) mbar_arrive(&sm->s_free[wg]);     // (the vote came after everybody's last read)
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->p_full[wg]);
            }
            // ---- the piece is done when the last products of both groups are
            if (wq == 0 && !gone && g_own < g_end) {
                const uint32_t last = g_end - 1u - ((g_end - 1u - g_own) & 1u);
                if (!mbar_wait(&sm->pv_done[wg], (last >> 1) & 1u, abort_flag, hdr, 44)) failed = true;
            }
            if (soft_sync_any(failed || gone)) break;
            tc_fence_after();
            const bool whole = s.cnt == s.T;
            const int slot = 2 * (int)blockIdx.x + (t > t_begin ? 1 : 0);
            const bool has0 = s.cnt > 1 || !(g_piece & 1u), has1 = s.cnt > 1 || (g_piece & 1u);   // groups with a tile in the piece
            const int* rows = sm->row[seg & 1u];
            // weights of the groups' accumulators, one thread per column (the sums of query r lie in lane r)
            if (wg == 0 && wq < (QB + 31) / 32) {
                const float l0 = tc_ld1(lane_addr + Col::L), l1 = tc_ld1(lane_addr + Col::L + 16);
                tc_wait_ld();
                if (r < 8 * n8) {
                    const float m0 = has0 ? -sm->nref[0][r] : -1e30f, m1 = has1 ? -sm->nref[1][r] : -1e30f, M = fmaxf(m0, m1);
                    float w0 = has0 ? exp2f(m0 - M) : 0.f, w1 = has1 ? exp2f(m1 - M) : 0.f;
                    const float sum = (has0 ? l0 * w0 : 0.f) + (has1 ? l1 * w1 : 0.f);
                    if (whole) {
                        const float inv = sum != 0.f ? 1.f / sum : 0.f;
                        w0 *= inv;
                        w1 *= inv;
                    } else {
                        p.part_ml[((size_t)slot * 2 + 0) * kWideQ + r] = M;
                        p.part_ml[((size_t)slot * 2 + 1) * kWideQ + r] = sum;
                    }
                    sm->alpha[0][r] = w0;
                    sm->alpha[1][r] = w1;
                }
            }
            soft_sync_any(false);
            // every other column group for each group of warps; thread r has channel r of both accumulators
#pragma unroll 1
            for (int j = wg; j < n8; j += 2) {
                float o[8], o1[8];
                if (has0) tc_ld8(lane_addr + Col::O + 8 * j, o);
                if (has1) tc_ld8(lane_addr + Col::O + QB + 8 * j, o1);
                float w0[8], w1[8];
                int row[8];
#pragma unroll
                for (int k = 0; k < 8; k += 4) {
                    *reinterpret_cast<float4*>(w0 + k) = *reinterpret_cast<const float4*>(&sm->alpha[0][8 * j + k]);
                    *reinterpret_cast<float4*>(w1 + k) = *reinterpret_cast<const float4*>(&sm->alpha[1][8 * j + k]);
                    *reinterpret_cast<int4*>(row + k) = *reinterpret_cast<const int4*>(rows + 8 * j + k);
                }
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = has0 ? o[k] * w0[k] : 0.f;
                    o[k] = has1 ? fmaf(o1[k], w1[k], x) : x;
                }
                if (whole) {
                    __nv_bfloat16* const out = p.out + r;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (8 * j + k < s.Nq) out[(size_t)(uint32_t)row[k] * kD] = __float2bfloat16_rn(o[k]);
                } else {
                    float* po = p.part_o + ((size_t)slot * kWideQ + 8 * j) * kD + r;
#pragma unroll
                    for (int k = 0; k < 8; ++k) po[k * kD] = o[k];
                }
            }
            if (!whole) __threadfence();
            tc_fence_before();
            soft_sync_any(false);                                // references, rows and accumulators have been read
            if (lane == 0) mbar_arrive(&sm->piece_done[seg & 1u]);
            t += s.cnt;
            g_piece = g_end;
        }
    }

    // ---- tear-down
    tc_fence_before();
    __syncthreads();
    if (warp == kScoreWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
    // ---- cut items that this block finished: four warps per column group, thread r channel r, pieces in block order
    if (sm->abort_flag) return;
#pragma unroll 1
    for (int x = 0; x < 2 * (QB / 8); ++x) {
        const auto& m = sm->merge[x & 1];
        const int j = x >> 1, r = tid & 127;
        if (j % (kThreads / 128) != tid >> 7 || m.T == 0 || m.before + m.cnt != m.T || 8 * j >= m.Nq) continue;
        __threadfence();
        // the pieces lie in consecutive blocks from block0 on, this one among them
        const int c0 = m.block0;
        int c1 = blockIdx.x + 1;
        while (c1 < pl.blocks && pl.first[c1] < m.first + m.T) ++c1;
        float M[8], l[8], o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) { M[k] = -INFINITY; l[k] = 0.f; o[k] = 0.f; }
#pragma unroll 2
        for (int c = c0; c < c1; ++c) {
            const long long a = pl.first[c];
            if (a == pl.first[c + 1]) continue;                  // a block without tiles
            const int sl = 2 * c + (a < m.first ? 1 : 0);
            const float* ml = p.part_ml + (size_t)sl * 2 * kWideQ + 8 * j;
            const float* po = p.part_o + ((size_t)sl * kWideQ + 8 * j) * kD + r;
            float mx[8], lx[8], ox[8];
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const float4 a4 = __ldcg(reinterpret_cast<const float4*>(ml + k)), b4 = __ldcg(reinterpret_cast<const float4*>(ml + kWideQ + k));
                mx[k] = a4.x; mx[k + 1] = a4.y; mx[k + 2] = a4.z; mx[k + 3] = a4.w;
                lx[k] = b4.x; lx[k + 1] = b4.y; lx[k + 2] = b4.z; lx[k + 3] = b4.w;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) ox[k] = __ldcg(po + k * kD);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float top = fmaxf(M[k], mx[k]), w0 = ex2_approx(M[k] - top), w1 = ex2_approx(mx[k] - top);
                l[k] = l[k] * w0 + lx[k] * w1;
                o[k] = o[k] * w0 + ox[k] * w1;
                M[k] = top;
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (8 * j + k < m.Nq) {
                const int q = m.q0 + 8 * j + k, n = q / p.G, h = m.hk * p.G + (q - n * p.G);
                p.out[(((size_t)m.b * p.Hkv * p.G + h) * p.N + n) * kD + r] = __float2bfloat16_rn(l[k] != 0.f ? o[k] * __frcp_rn(l[k]) : 0.f);
            }
        }
    }
}

template <int QB>
int launch(const Params& p, int grid, cudaStream_t stream) {
    constexpr size_t smem_bytes = 1024 + 6 * QB * 256 + (size_t)kStages<QB> * kStageBytes + sizeof(Small<QB>);
    static_assert(smem_bytes <= kSmemLimit, "ring and buffers fit the block's shared memory");
    static std::mutex mu;                                        // the opt-in to large shared memory is per device
    static bool done[64] = {};
    int dev = 0;
    MCSD_CUDA_CHECK(cudaGetDevice(&dev));
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev < 0 || dev >= 64 || !done[dev]) {
            MCSD_CUDA_CHECK(cudaFuncSetAttribute(tree_attention_kv4_kernel<QB>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
            if (dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see the kernel's set-up
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, tree_attention_kv4_kernel<QB>, p));
    count_launches(1);
    return MCSD_OK;
}

constexpr size_t kMlBytes = (size_t)2 * kMaxCtas * 2 * kWideQ * sizeof(float);
constexpr size_t kOBytes = (size_t)2 * kMaxCtas * kWideQ * kD * sizeof(float);

}  // namespace

// The shapes of the tensor-core kernel over dense caches, as long as the tiles of one sequence can be counted in 31 bits.
bool kv4_tc_shape(int B, int H, int G, int N, int D, int L_max, int dtype) {
    const long long blocks_q = ((long long)G * N + kWideQ - 1) / kWideQ;
    return tc_shape_supported(B, H, G, N, D, L_max, dtype) && (H / G) * blocks_q * ((long long)L_max / kTile + 4) < (1LL << 31);
}

size_t kv4_tc_workspace_bytes() { return kMlBytes + kOBytes; }

int tree_attention_kv4_tc(const AttentionArgs& a, AttentionWorkspace* workspace, void* scratch, cudaStream_t stream) {
    static thread_local int sms_dev = -1, sms = 0;
    int dev = 0;
    MCSD_CUDA_CHECK(cudaGetDevice(&dev));
    if (sms_dev != dev) {
        MCSD_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        sms_dev = dev;
    }
    Params p;
    p.q = static_cast<const __nv_bfloat16*>(a.q);
    p.k_tree = static_cast<const __nv_bfloat16*>(a.k_tree);
    p.v_tree = static_cast<const __nv_bfloat16*>(a.v_tree);
    p.cache = static_cast<const unsigned char*>(a.kv4);
    p.out = static_cast<__nv_bfloat16*>(a.out);
    p.seq_lens = a.seq_lens;
    p.n_active = a.n_active;
    p.anc = a.anc;
    p.words = a.words;
    p.B = a.B; p.Hkv = a.H / a.G; p.G = a.G; p.N = a.N; p.pages = a.L_max / kPageRows;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.part_ml = static_cast<float*>(scratch);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(scratch) + kMlBytes);
    p.counters = workspace->counters;
    p.header = &workspace->header;
    const int grid = std::min(sms, kMaxCtas);
    // Few query columns (single tokens): the smaller kernel starts and merges faster, 15.6 against 16.4 us for one token after 1001
    // rows, 67 us either way for 8 x 32001 (with room for a sixth tile).  Another one for 48 columns brought nothing.
    if (a.N * a.G <= 16) return launch<16>(p, grid, stream);
    return launch<kWideQ>(p, grid, stream);
}

}  // namespace mcsd
