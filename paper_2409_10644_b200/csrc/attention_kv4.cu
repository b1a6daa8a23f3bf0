// Tree attention (Section 2.2 of the paper) over a prefix cache held in 4 bits (page layout in kv4.cuh), on the
// fifth-generation tensor cores of sm_100a: bf16 tree tensors, head_dim 128, 1 to 64 query columns per work item.
//
// The products are set up transposed, the small dimension (query columns) as the MMA N:
//     S^T[key][query] = K Q^T,     O^T[channel][query] += V^T P^T,     l[query] += 1 P^T
// and the A operands live in tensor memory, not in shared memory: thread r of the key warps owns key row r of a
// 128-key tile, thread d of the value warps channel d, and both turn 16-byte pieces of a page (neighbouring threads read
// neighbouring pieces) into operand columns with a shift and a mask per two values and store them with tcgen05.st.
//   * Keys stay codes: 16 + code is exact in bf16, so S' = sum (16 + code) q is exact up to fp32 sums, and the row's scale
//     and offset are applied to the score, where the softmax thread owns the same key row:
//         score = scale_k S' + offset_k (sum of q).
//   * Values become scale_v (16 + code) + offset_v, one packed fused multiply-add per two values.  They and the weights
//     that multiply them are fp16 (11 bits: an order of magnitude below the rounding of the bf16 result) in every tile
//     whose values lie well inside fp16's range, which the value warps vote on tile by tile; else bf16.
// The rows of the tree itself are read as they are (bf16): same operand columns, scale 1, offset 0.
//
// What bounds it: 136 bytes per key and head against 512 in bf16 move the floor of a launch down by 3.8; unpacking
// and the exponentials then share the issue slots of the schedulers, so the work is spread over specialised warps:
//   warps 0-3    keys      page pieces -> operand columns
//   warps 4-7    values    page pieces -> operand columns
//   warps 8-11   softmax of the even tiles, all columns;  warps 12-15 of the odd ones.  The two groups have their own
//                references, accumulators and row sums and meet only at the end of a work item: with one group per tile
//                a tile's chain (scores, vote, exponentials, P^T, products) may take twice the time between two tiles
//   warp 16      copies whole pages (1 to 4 of them, contiguous) into a ring with cp.async.bulk
//   warp 17      issues the MMAs and owns the tensor memory
//   warps 18-19  bring the queries of the next work item and their sums
// Loops are rolled as far as the latencies allow: the roles share the instruction caches, and with unrolled bodies (a
// kernel of 180 KB) a tile took three times as long, most of it in waits for instructions.
//
// Work: one block per multiprocessor walks a contiguous range of the (sequence, key/value head, query block, tile) space,
// cut by cost.  A work item that a range boundary cuts is finished by whichever of its blocks comes last (a counter of
// tiles per item; nothing waits): it reads all pieces in block order, so the result does not depend on who that is.
// Every wait is bounded; one that runs out raises a flag in the workspace header.
#include <algorithm>
#include <mutex>
#include <type_traits>

#include <cuda_fp16.h>

#include "attention_tc_common.cuh"
#include "kv4.cuh"

namespace mcsd {

namespace {

constexpr int kD = 128;
constexpr int kPageBytes = kv4_page_bytes(kD);
constexpr int kStageBytes = 4 * kPageBytes;      // one tile: 128 rows
constexpr int kValueWarp = 4, kSoftWarp = 8, kCopyWarp = 16, kIssueWarp = 17, kQueryWarp = 18;
constexpr int kThreads = 640;
constexpr int kWideQ = 64;                       // query columns of a work item, at most
constexpr int kStages = 6;
constexpr int kMaxPieces = kMaxCtas;             // of a work item
// Tensor-memory columns: scores, O^T and row sums of the two softmax groups, then keys and values, twice where it fits,
// and the ones of the row sums' A operand (bf16, fp16; they are in shared memory where no column is left, and such a
// product takes 41 cycles instead of 12 at 16 columns, 50 instead of 34 at 64).
template <int QB>
struct Columns {
    static constexpr int S = 0, O = 2 * QB, L = 4 * QB, K = 6 * QB;
    static constexpr bool ones = K + 128 + 16 <= kTmemCols;
    static constexpr int key_buffers = K + 256 + 16 <= kTmemCols ? 2 : 1;
    static constexpr int V = K + 64 * key_buffers;
    static constexpr int value_buffers = V + 128 + 16 <= kTmemCols ? 2 : 1;
    static constexpr int One = V + 64 * value_buffers;
    static_assert(One + (ones ? 16 : 0) <= kTmemCols, "tensor memory");
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
    int* counters;        // [work items] tiles that have been finished; zero between launches
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

// Cost of a tile with nq query columns and of a work item on top of its tiles.
__host__ __device__ __forceinline__ int tile_cost(int nq) { return 32 + nq / 2; }
constexpr int kItemCost = 64;

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
    const long long x = (total * c + pl.blocks - 1) / pl.blocks;
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pl.cost[mid] <= x) lo = mid; else hi = mid;
    }
    const Shape sh = shape_of<QB>(pl.len[lo], pl.nodes[lo], p.G);
    if (sh.T == 0) return pl.tiles[p.B];
    const int w = tile_cost(sh.per_q);
    const long long ci = (long long)sh.T * w + kItemCost, off = x - pl.cost[lo];
    const long long it = off / ci, rem = off - it * ci;
    const long long lt = (rem + w - 1) / w;
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
    unsigned long long full[kStages], empty[kStages];
    unsigned long long k_full[2], s_full[2], s_free[2], v_full[2], p_full[2], pv_done[2], q_full[2], piece_done[2], fmt_full[4];
    unsigned long long drain;
    uint32_t tmem_base;
    int abort_flag;
    int merge, merge_pieces;                          // tiles of the item finished before this block's; its pieces
    int fmt[4];                                       // 1: the tile's values and weights are fp16, 0: bf16
    int row[2][QB];                                   // rows of q and out of the piece's columns
    short slots[kMaxPieces];                          // of the pieces that are merged
    alignas(16) float2 kab[4][kTile];                 // scale and offset of a tile's key rows, in score units
    alignas(16) unsigned short vab[2][2][kTile];      // scales and offsets of a tile's value rows, in the tile's format
    alignas(16) float q_sum[2][QB];
    alignas(16) float nref[2][QB];                    // running references of the two groups, negated
    alignas(16) float alpha[2][QB];
    alignas(16) float red[2][4][QB];
    alignas(16) uint64_t anc[MCSD_MAX_NODES * MCSD_MAX_WORDS];
    alignas(16) unsigned short ones[2][kTile * 16];   // A operand of the row sums: bf16, fp16
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
// codes (2i, 2i + 1) of a word as two numbers 16 + code: bf16 (code in mantissa bits 3..6) or fp16 (bits 6..9)
template <bool HALF>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i) {
    if (HALF) {
        const uint32_t x = i < 2 ? w << (6 - 4 * i) : w >> (4 * i - 6);
        return (x & 0x03C003C0u) | 0x4C004C00u;
    }
    const uint32_t x = i == 0 ? w << 3 : w >> (4 * i - 3);
    return (x & 0x00780078u) | 0x41804180u;
}
template <bool HALF>
__device__ __forceinline__ uint32_t fma_x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    if (HALF) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    uint32_t d;
    if (HALF) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// two fp32 fused multiply-adds in one instruction
__device__ __forceinline__ float2 fma_f32x2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
// barrier over both softmax groups
__device__ __forceinline__ bool both_sync_any(bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.or.pred q, 4, 256, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r) : "r"((uint32_t)pred) : "memory");
    return r != 0;
}
// A row of values may be fp16: no value can leave its range, and neither scale nor values are so small that fp16's fixed
// spacing below 2^-14 would round them more coarsely than bf16 does.  False for scales that are not finite.
__device__ __forceinline__ bool fits_half(float scale, float offset) {
    const float o = fabsf(offset);
    return 31.f * scale + o <= 32768.f && (scale >= 6.103515625e-5f || (scale == 0.f && (o == 0.f || o >= 6.103515625e-5f)));
}

template <int QB>
__global__ void __launch_bounds__(kThreads, 1)
tree_attention_kv4_kernel(const Params p) {
    using Col = Columns<QB>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);   // (an offset: the compiler keeps knowing it is shared memory)
    unsigned char* q_buf = smem;                      // two buffers of QB rows: [2 slabs of 64 channels][QB rows][128 bytes], swizzled
    unsigned char* p_buf = q_buf + 2 * QB * 256;      // P^T of the two groups: [QB / 8][128 keys][16 bytes]
    unsigned char* ring = p_buf + 2 * QB * 256;
    Small<QB>* sm = reinterpret_cast<Small<QB>*>(ring + kStages * kStageBytes);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- set-up; what comes before the wait touches no global memory and overlaps the tail of the preceding kernel
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&sm->full[i], 1); mbar_init(&sm->empty[i], 8); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm->k_full[i], 4);
            mbar_init(&sm->s_full[i], 1);
            mbar_init(&sm->s_free[i], 4);
            mbar_init(&sm->v_full[i], 4);
            mbar_init(&sm->p_full[i], 4);
            mbar_init(&sm->pv_done[i], 1);
            mbar_init(&sm->q_full[i], 2);
            mbar_init(&sm->piece_done[i], 8);
        }
        for (int i = 0; i < 4; ++i) mbar_init(&sm->fmt_full[i], 4);
        mbar_init(&sm->drain, 1);
        sm->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < kTile * 16; i += kThreads) { sm->ones[0][i] = 0x3F80; sm->ones[1][i] = 0x3C00; }
    fence_async_smem();                               // read by the tensor cores through the async proxy
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = tid; i < p.N * p.words; i += kThreads) sm->anc[i] = p.anc[i];
    make_plan<QB>(sm->plan, p);
    const Plan& pl = sm->plan;
    const long long t_begin = pl.first[blockIdx.x], t_end = pl.first[blockIdx.x + 1];
    if (t_begin >= t_end) return;                     // uniform for the whole block: nothing allocated yet

    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t*)&sm->tmem_base;
    WorkspaceHeader* const hdr = p.header;
    int* const abort_flag = &sm->abort_flag;

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
                for (int i = s.lt; i < min(s.lt + s.cnt, s.Tp) && ok; ++i, ++f) {
                    const uint32_t st = f % kStages;
                    if (f >= kStages) ok = mbar_wait(&sm->empty[st], (f / kStages - 1u) & 1u, abort_flag, hdr, 31);
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
                for (uint32_t x = f > kStages ? f - kStages : 0; x < f; ++x) {
                    const long long t0 = clock64();
                    while (!mbar_try_wait(&sm->full[x % kStages], (x / kStages) & 1u) && clock64() - t0 < kSpinCycles / 8) {}
                }
            }
        }
    } else if (warp == kIssueWarp) {
        // S^T of tile g + 1 is issued before the products of tile g, across pieces as well
        const uint64_t dq0 = smem_desc(smem_u32(q_buf), 16, 1024, 2);
        const uint64_t dp0 = smem_desc(smem_u32(p_buf), 128, 2048, 0);
        const uint64_t d1 = smem_desc(smem_u32(sm->ones), 128, 256, 0);
        constexpr uint32_t q_slab = (QB * 128) >> 4, q_next = (QB * 256) >> 4, p_next = (QB * 256) >> 4, one_next = (kTile * 32) >> 4;
        const uint32_t n_tiles = (uint32_t)(t_end - t_begin);
        Piece s;                                      // of the scores
        long long ts = t_begin;
        int si = 0, oi = 0, o_cnt = 0, o_nq = 0;      // the products are one tile behind: in the same piece or the one before
        uint32_t seg = 0;
        bool ok = true;
        s.cnt = 0;
        for (uint32_t g = 0; g <= n_tiles && ok; ++g) {
            if (g < n_tiles) {
                if (si == s.cnt) {
                    ts += s.cnt;
                    piece_at<QB>(pl, p, ts, t_end, s);
                    si = 0;
                    ok = mbar_wait(&sm->q_full[seg & 1u], (seg >> 1) & 1u, abort_flag, hdr, 32);
                    if (!ok) break;
                    ++seg;
                }
                const uint32_t buf = g & 1u;
                ok = mbar_wait(&sm->k_full[buf], (g >> 1) & 1u, abort_flag, hdr, 33);
                if (ok && g >= 2) ok = mbar_wait(&sm->s_free[buf], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 46);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t idesc = instr_desc((s.Nq + 15) & ~15, 0, 0);
                    const uint64_t dq = dq0 + ((seg - 1u) & 1u) * q_next;
                    const uint32_t d = tmem + Col::S + buf * QB, ka = tmem + Col::K + (Col::key_buffers == 2 ? buf * 64 : 0u);
#pragma unroll
                    for (int k = 0; k < 8; ++k) mma_ta(d, ka + 8 * k, dq + (uint32_t)(k >> 2) * q_slab + (uint32_t)(k & 3) * 2u, idesc, k > 0);
                    commit(&sm->s_full[buf]);
                }
                __syncwarp();
                ++si;
            }
            if (g >= 1) {
                const uint32_t h = g - 1u, hb = h & 1u;
                ok = mbar_wait(&sm->v_full[hb], (h >> 1) & 1u, abort_flag, hdr, 34);
                if (ok) ok = mbar_wait(&sm->p_full[hb], (h >> 1) & 1u, abort_flag, hdr, 35);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    // fp16 operands are format 0 of both operand fields, bf16 is 1
                    const uint32_t half = sm->fmt[h & 3u];
                    const uint32_t idesc = instr_desc((o_nq + 15) & ~15, 0, 1) & ~(half ? (1u << 7) | (1u << 10) : 0u);
                    const uint32_t d = tmem + Col::O + hb * QB, l = tmem + Col::L + hb * QB;
                    const uint32_t va = tmem + Col::V + (Col::value_buffers == 2 ? hb * 64 : 0u), one = tmem + Col::One + half * 8;
                    const uint64_t dp = dp0 + hb * p_next, d1h = d1 + half * one_next;
                    const uint32_t more = oi >= 2;    // a group's first tile of a piece overwrites
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        mma_ta(d, va + 8 * k, dp + (uint32_t)(k * (256 >> 4)), idesc, more | (uint32_t)(k > 0));
                        if (Col::ones) mma_ta(l, one, dp + (uint32_t)(k * (256 >> 4)), idesc, more | (uint32_t)(k > 0));
                        else mma_sa(l, d1h, dp + (uint32_t)(k * (256 >> 4)), idesc, more | (uint32_t)(k > 0));
                    }
                    commit(&sm->pv_done[hb]);
                }
                __syncwarp();
                ++oi;
            }
            if (oi == o_cnt) { oi = 0; o_cnt = s.cnt; o_nq = s.Nq; }   // the next products belong to the scores' piece
        }
        if (elect_one()) commit(&sm->drain);          // all MMAs have finished before tensor memory is released
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&sm->drain, 0) && clock64() - t0 < kSpinCycles) {}
    } else if (warp >= kQueryWarp) {
        // Queries of the next piece: sixteen lanes per row, 16 bytes each, into the swizzled operand layout; rows past the
        // last query are zeros.  Stacked query j of a key/value head is head j % G of its group, node j / G.
        const int sub = lane >> 4, c = lane & 15;
        uint32_t seg = 0;
        for (long long t = t_begin; t < t_end; ++seg) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            const uint32_t buf = seg & 1u;
            if (seg >= 2 && !mbar_wait(&sm->piece_done[buf], ((seg - 2u) >> 1) & 1u, abort_flag, hdr, 36)) break;
            const int rows = (s.Nq + 15) & ~15;
            unsigned char* dst = q_buf + buf * (QB * 256) + (c >> 3) * (QB * 128);
#pragma unroll 4
            for (int r = (warp - kQueryWarp) * 2 + sub; r < rows; r += 4) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (r < s.Nq) {
                    const int j = s.q0 + r, n = j / p.G, h = s.hk * p.G + (j - n * p.G);
                    const int row = (s.b * p.Hkv * p.G + h) * p.N + n;          // below 65535 * 192
                    v = *reinterpret_cast<const uint4*>(p.q + (size_t)row * kD + c * 8);
                    if (c == 0) sm->row[buf][r] = row;
                }
                *reinterpret_cast<uint4*>(dst + r * 128 + (((c & 7) ^ (r & 7)) * 16)) = v;
                float sum = 0.f;
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += __uint_as_float(w[i] << 16) + __uint_as_float(w[i] & 0xFFFF0000u);
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                if (c == 0) sm->q_sum[buf][r] = sum;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm->q_full[buf]);
            t += s.cnt;
        }
    } else if (warp < kValueWarp) {
        // ---- keys: thread r owns key row r of a tile
        constexpr uint32_t NK = Col::key_buffers;
        const int r = tid;
        const uint32_t lane_addr = tmem + ((uint32_t)(warp * 32) << 16);
        if (Col::ones) {                              // ordered before the products by the barrier of the first tile's keys
            uint32_t y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = e < 8 ? 0x3F803F80u : 0x3C003C00u;
            tc_st16(lane_addr + Col::One, y);
        }
        uint32_t g = 0, f = 0;
        bool ok = true;
        for (long long t = t_begin; t < t_end && ok;) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            for (int i = s.lt; i < s.lt + s.cnt && ok; ++i, ++g) {
                const uint32_t buf = g & 1u, dst = lane_addr + Col::K + (NK == 2 ? buf * 64 : 0u);
                if (i < s.Tp) {
                    const uint32_t st = f % kStages;
                    ok = mbar_wait(&sm->full[st], (f / kStages) & 1u, abort_flag, hdr, 37);
                    if (!ok) break;
                    const unsigned char* page = ring + st * kStageBytes + warp * kPageBytes;   // rows 32 warp .. of the tile
                    const uint4* piece = reinterpret_cast<const uint4*>(page) + lane;
                    const unsigned short* sc = reinterpret_cast<const unsigned short*>(page + kv4_scales_at(kD));
                    const float a = bf16_bits_to_f32(sc[lane]), b = bf16_bits_to_f32(sc[kPageRows + lane]);
                    uint4 x = piece[0];
                    // The buffer is free once the scores of the tile that used it are done.  They were issued after the
                    // softmax warps had taken the scores and the scales of tile g - 4, which the entry below held.
                    if (g >= NK) ok = mbar_wait(&sm->s_full[(g - NK) & 1u], ((g - NK) >> 1) & 1u, abort_flag, hdr, 38);
                    if (!ok) break;
                    tc_fence_after();
                    sm->kab[g & 3u][r] = make_float2(a * p.scale_log2, b * p.scale_log2);
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        const uint4 next = piece[((c + 1) & 3) * kPageRows];
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                        uint32_t y[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = code_pair<false>(w[e >> 2], e & 3);
                        tc_st16(dst + 16 * c, y);
                        x = next;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->empty[st]);
                    ++f;
                } else {
                    const int n = (i - s.Tp) * kTile + r;
                    if (g >= NK) ok = mbar_wait(&sm->s_full[(g - NK) & 1u], ((g - NK) >> 1) & 1u, abort_flag, hdr, 38);
                    if (!ok) break;
                    tc_fence_after();
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
                        tc_st16(dst + 16 * c, y);
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
        constexpr uint32_t NV = Col::value_buffers;
        const int d = tid & 127;
        const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + Col::V;
        uint32_t g = 0, f = 0;
        bool failed = false, gone = false;                    // gone: all threads of the role know that one has failed
        for (long long t = t_begin; t < t_end && !gone;) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            for (int i = s.lt; i < s.lt + s.cnt; ++i, ++g) {
                const uint32_t dst = lane_addr + (NV == 2 ? (g & 1u) * 64 : 0u);
                const uint32_t st = f % kStages;
                unsigned short* const va = sm->vab[g & 1u][0];
                unsigned short* const vb = sm->vab[g & 1u][1];
                uint32_t a16 = 0, b16 = 0;
                if (i < s.Tp) {
                    if (!mbar_wait(&sm->full[st], (f / kStages) & 1u, abort_flag, hdr, 39)) failed = true;
                    // Scales of the tile's rows, thread d the row d, rounded to fp16.  Rows past the end of the prefix have
                    // probability zero but may hold anything, and 0 * NaN would be NaN: their scale and offset are zero.
                    const unsigned short* sc = reinterpret_cast<const unsigned short*>(ring + st * kStageBytes + (warp & 3) * kPageBytes + kv4_scales_at(kD)) + 2 * kPageRows + lane;
                    if (d < s.L - i * kTile) { a16 = sc[0]; b16 = sc[kPageRows]; }
                    va[d] = __half_as_ushort(__float2half_rn(bf16_bits_to_f32(a16)));
                    vb[d] = __half_as_ushort(__float2half_rn(bf16_bits_to_f32(b16)));
                }
                const bool half = !group_sync_any(3, failed || i >= s.Tp || !fits_half(bf16_bits_to_f32(a16), bf16_bits_to_f32(b16)));
                if (!half) {
                    va[d] = (unsigned short)a16;
                    vb[d] = (unsigned short)b16;
                    gone = group_sync_any(3, failed);
                    if (gone) break;
                }
                if (lane == 0) {
                    if (warp == kValueWarp) sm->fmt[g & 3u] = half;
                    mbar_arrive(&sm->fmt_full[g & 3u]);
                }
                // the buffer is free once the products of the tile that used it are done
                if (g >= NV && !mbar_wait(&sm->pv_done[(g - NV) & 1u], ((g - NV) >> 1) & 1u, abort_flag, hdr, 40)) failed = true;
                tc_fence_after();
                if (i < s.Tp) {
                    const unsigned char* codes = ring + st * kStageBytes + kv4_values_at(kD) + d * 16;
                    const uint4* sa = reinterpret_cast<const uint4*>(va);
                    const uint4* sb = reinterpret_cast<const uint4*>(vb);
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
        // ---- softmax, epilogue, merge: group wg has the tiles with g % 2 == wg, thread r key row r
        const int wg = (warp - kSoftWarp) >> 2, wq = warp & 3, r = tid & 127;
        const int bar_id = 1 + wg;
        const uint32_t lane_addr = tmem + ((uint32_t)(wq * 32) << 16);
        unsigned char* const p_own = p_buf + wg * (QB * 256) + r * 16;
        float* const nref = sm->nref[wg];
        uint32_t g_piece = 0, seg = 0;                           // tiles of this block before the piece
        bool failed = false, gone = false;                       // gone: all threads know that one has failed
        for (long long t = t_begin; t < t_end; ++seg) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            const int n8 = (s.Nq + 7) >> 3;
            const float* qs = sm->q_sum[seg & 1u];
            const uint32_t g_end = g_piece + (uint32_t)s.cnt;
            const uint32_t g_own = g_piece + ((g_piece ^ (uint32_t)wg) & 1u);   // the group's first tile, if below g_end
            for (uint32_t g = g_own; g < g_end; g += 2) {
                const int i = s.lt + (int)(g - g_piece);
                const bool tree = i >= s.Tp;
                const int key = (tree ? i - s.Tp : i) * kTile + r;
                const bool plain = !tree && (i + 1) * kTile <= s.L;   // every key there and visible to every query
                unsigned long long cm = 0;                       // columns that see this thread's key
                if (!plain) {
                    if (!tree) {
                        if (key < s.L) cm = ~0ull;
                    } else if (key < s.Nb) {
                        int n = s.q0 / p.G, rest = s.q0 - n * p.G;
                        for (int c = 0; c < s.Nq; ++c) {
                            cm |= (unsigned long long)((sm->anc[n * p.words + (key >> 6)] >> (key & 63)) & 1ull) << c;
                            if (++rest == p.G) { rest = 0; ++n; }
                        }
                    }
                }
                if (!mbar_wait(&sm->s_full[wg], (g >> 1) & 1u, abort_flag, hdr, 41)) failed = true;
                if (!mbar_wait(&sm->fmt_full[g & 3u], (g >> 2) & 1u, abort_flag, hdr, 45)) failed = true;
                // P^T is free once the products of the group's previous tile are done, and the accumulators are current
                if (g >= 2 && !mbar_wait(&sm->pv_done[wg], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 43)) failed = true;
                tc_fence_after();
                const bool half = sm->fmt[g & 3u], first = g == g_own;
                const float2 ab = sm->kab[g & 3u][r];
                const float2 a2 = make_float2(ab.x, ab.x), b2 = make_float2(ab.y, ab.y);
                const uint32_t s_addr = lane_addr + Col::S + wg * QB;
                // New references come first in a piece's first tile, and again where a score exceeds its reference by more
                // than 2^8 after the optimistic sweep below, which is then redone.
                bool raise = first, raised = false;
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
                        if (r < 8 * n8) {
                            const float top = fmaxf(fmaxf(sm->red[wg][0][r], sm->red[wg][1][r]), fmaxf(sm->red[wg][2][r], sm->red[wg][3][r]));
                            // (a column that has seen no key yet keeps one below any score)
                            const float old = first ? -1e30f : -nref[r], now = fmaxf(old, top);
                            nref[r] = -now;
                            sm->alpha[wg][r] = exp2f(old - now);
                        }
                        group_sync_any(bar_id, false);
                        if (!first) {
#pragma unroll 1
                            for (int j = 0; j < 2 * n8; ++j) {   // accumulators, then row sums
                                const int jj = j < n8 ? j : j - n8;
                                const uint32_t at = lane_addr + (j < n8 ? Col::O : Col::L) + wg * QB + 8 * jj;
                                float o[8];
                                tc_ld8(at, o);
                                tc_wait_ld();
#pragma unroll
                                for (int k = 0; k < 8; ++k) o[k] *= sm->alpha[wg][8 * jj + k];
                                tc_st8(at, o);
                            }
                            tc_wait_st();
                        }
                    }
                    // scores of this thread's key relative to the references, exponentiated, packed, stored: two column
                    // groups at a time (one is enough to keep the unit busy only with four times the warps)
                    float dmax = -INFINITY;
#pragma unroll 1
                    for (int j = 0; j < n8; j += 2) {
                        float y[2][8];
                        tc_ld8(s_addr + 8 * j, y[0]);
                        if (j + 1 < n8) tc_ld8(s_addr + 8 * j + 8, y[1]);
                        tc_wait_ld();
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (j + h < n8) {
                                const float* qj = qs + 8 * (j + h);
                                const float* nj = nref + 8 * (j + h);
#pragma unroll
                                for (int k = 0; k < 8; k += 4) {
                                    const float4 q = *reinterpret_cast<const float4*>(qj + k), m = *reinterpret_cast<const float4*>(nj + k);
                                    const float2 u = fma_f32x2(make_float2(y[h][k], y[h][k + 1]), a2, fma_f32x2(make_float2(q.x, q.y), b2, make_float2(m.x, m.y)));
                                    const float2 v = fma_f32x2(make_float2(y[h][k + 2], y[h][k + 3]), a2, fma_f32x2(make_float2(q.z, q.w), b2, make_float2(m.z, m.w)));
                                    y[h][k] = u.x; y[h][k + 1] = u.y; y[h][k + 2] = v.x; y[h][k + 3] = v.y;
                                }
                                if (!plain) {
                                    const uint32_t bits = (uint32_t)(cm >> (8 * (j + h)));
#pragma unroll
                                    for (int k = 0; k < 8; ++k) y[h][k] = ((bits >> k) & 1u) ? y[h][k] : -INFINITY;
                                }
                                dmax = fmaxf(dmax, fmaxf(fmaxf(fmaxf(y[h][0], y[h][1]), fmaxf(y[h][2], y[h][3])), fmaxf(fmaxf(y[h][4], y[h][5]), fmaxf(y[h][6], y[h][7]))));
                                uint32_t w[4];
#pragma unroll
                                for (int k = 0; k < 8; ++k) y[h][k] = ex2_approx(y[h][k]);
                                if (half) {
#pragma unroll
                                    for (int k = 0; k < 4; ++k) w[k] = pack_pair<true>(y[h][2 * k], y[h][2 * k + 1]);
                                } else {
#pragma unroll
                                    for (int k = 0; k < 4; ++k) w[k] = pack_pair<false>(y[h][2 * k], y[h][2 * k + 1]);
                                }
                                *reinterpret_cast<uint4*>(p_own + (j + h) * 2048) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                    raise = group_sync_any(bar_id, (dmax > kLazyTau && !raised) || failed);   // one vote of the group
                    if (!raise) break;
                    gone = group_sync_any(bar_id, failed);
                    if (gone) break;
                }
                if (gone) break;
                tc_fence_before();
                if (lane == 0) mbar_arrive(&sm->s_free[wg]);     // (the vote above came after everybody's last read)
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->p_full[wg]);
            }
            // ---- the piece is done when the last products of both groups are
            if (!gone && g_own < g_end) {
                const uint32_t last = g_end - 1u - ((g_end - 1u - g_own) & 1u);
                if (!mbar_wait(&sm->pv_done[wg], (last >> 1) & 1u, abort_flag, hdr, 44)) failed = true;
            }
            if (both_sync_any(failed || gone)) break;
            tc_fence_after();
            const bool whole = s.cnt == s.T;
            const int slot = 2 * (int)blockIdx.x + (t > t_begin ? 1 : 0);
            const bool has0 = s.cnt > 1 || !(g_piece & 1u), has1 = s.cnt > 1 || (g_piece & 1u);   // groups with a tile in the piece
            const int* rows = sm->row[seg & 1u];
            // the groups split the columns; thread r has channel r of both accumulators
            const int j0 = wg ? (n8 + 1) / 2 : 0, j1 = wg ? n8 : (n8 + 1) / 2;
#pragma unroll 1
            for (int j = j0; j < j1; ++j) {
                float o0[8], o1[8], l0[8], l1[8];
                tc_ld8(lane_addr + Col::O + 8 * j, o0);
                tc_ld8(lane_addr + Col::O + QB + 8 * j, o1);
                tc_ld8(lane_addr + Col::L + 8 * j, l0);
                tc_ld8(lane_addr + Col::L + QB + 8 * j, l1);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int c = 8 * j + k;
                    if (c < s.Nq) {
                        const float m0 = has0 ? -sm->nref[0][c] : -1e30f, m1 = has1 ? -sm->nref[1][c] : -1e30f, M = fmaxf(m0, m1);
                        const float w0 = ex2_approx(m0 - M), w1 = ex2_approx(m1 - M);
                        const float o = (has0 ? o0[k] * w0 : 0.f) + (has1 ? o1[k] * w1 : 0.f);
                        const float l = (has0 ? l0[k] * w0 : 0.f) + (has1 ? l1[k] * w1 : 0.f);
                        if (whole) {
                            p.out[(size_t)rows[c] * kD + r] = __float2bfloat16_rn(l != 0.f ? o / l : 0.f);
                        } else {
                            p.part_o[((size_t)slot * kWideQ + c) * kD + r] = o;
                            if (r == 0) {
                                p.part_ml[((size_t)slot * 2 + 0) * kWideQ + c] = M;
                                p.part_ml[((size_t)slot * 2 + 1) * kWideQ + c] = l;
                            }
                        }
                    }
                }
            }
            if (!whole) {
                // the block that finishes an item's last tile merges all pieces
                __threadfence();
                both_sync_any(false);
                const long long first = pl.tiles[s.b] + (long long)(s.item - pl.items[s.b]) * s.T;   // the item's first tile
                if (tid == kSoftWarp * 32) sm->merge = atomicAdd(&p.counters[s.item], s.cnt);
                // every block's piece of this item: its slot, or -1
                const int c = tid - kSoftWarp * 32;
                if (c < pl.blocks) {
                    const long long a = pl.first[c], b = pl.first[c + 1];
                    sm->slots[c] = max(a, first) < min(b, first + s.T) ? (short)(2 * c + (a < first ? 1 : 0)) : (short)-1;
                }
                both_sync_any(false);
                if (sm->merge + s.cnt == s.T) {
                    __threadfence();
                    // the item's pieces lie in consecutive blocks, this one among them
                    int c0 = blockIdx.x, c1 = blockIdx.x + 1;
                    while (c0 > 0 && pl.first[c0] > first) --c0;
                    while (c1 < pl.blocks && pl.first[c1] < first + s.T) ++c1;
#pragma unroll 1
                    for (int j = j0; j < j1; ++j) {
                        float M[8], l[8], o[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) { M[k] = -INFINITY; l[k] = 0.f; o[k] = 0.f; }
#pragma unroll 1
                        for (int x = c0; x < c1; ++x) {
                            const int sl = sm->slots[x];
                            if (sl < 0) continue;
                            const float* ml = p.part_ml + (size_t)sl * 2 * kWideQ + 8 * j;
                            const float* po = p.part_o + ((size_t)sl * kWideQ + 8 * j) * kD + r;
                            float mx[8], lx[8], ox[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (8 * j + k < s.Nq) { mx[k] = __ldcg(ml + k); lx[k] = __ldcg(ml + kWideQ + k); ox[k] = __ldcg(po + k * kD); }
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                if (8 * j + k < s.Nq) {
                                    const float m = fmaxf(M[k], mx[k]), w0 = ex2_approx(M[k] - m), w1 = ex2_approx(mx[k] - m);
                                    l[k] = l[k] * w0 + lx[k] * w1;
                                    o[k] = o[k] * w0 + ox[k] * w1;
                                    M[k] = m;
                                }
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (8 * j + k < s.Nq) p.out[(size_t)rows[8 * j + k] * kD + r] = __float2bfloat16_rn(l[k] != 0.f ? o[k] / l[k] : 0.f);
                    }
                    if (tid == kSoftWarp * 32) p.counters[s.item] = 0;
                }
            }
            tc_fence_before();
            both_sync_any(false);                                // references, rows and accumulators have been read
            if (lane == 0) mbar_arrive(&sm->piece_done[seg & 1u]);
            t += s.cnt;
            g_piece = g_end;
        }
    }

    // ---- tear-down
    tc_fence_before();
    __syncthreads();
    if (warp == kIssueWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// Query columns a launch is built for: all of them when they fit one block, else the even share of the fewest blocks.
int columns_for(int nq) {
    const int blocks = (nq + kWideQ - 1) / kWideQ;
    const int per = ((nq + blocks - 1) / blocks + 7) & ~7;
    return per <= 16 ? 16 : per <= 32 ? 32 : per <= 48 ? 48 : kWideQ;
}

template <int QB>
int launch(const Params& p, int grid, cudaStream_t stream) {
    constexpr size_t smem_bytes = 1024 + 4 * QB * 256 + (size_t)kStages * kStageBytes + sizeof(Small<QB>);
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

size_t kv4_tc_workspace_bytes(int B, int H, int G, int N) {
    const size_t blocks_q = ((size_t)G * N + kWideQ - 1) / kWideQ;
    return kMlBytes + kOBytes + align_up((size_t)B * (H / G) * blocks_q * sizeof(int), 256);
}

int tree_attention_kv4_tc(const AttentionArgs& a, WorkspaceHeader* header, void* scratch, cudaStream_t stream) {
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
    p.counters = reinterpret_cast<int*>(static_cast<char*>(scratch) + kMlBytes + kOBytes);
    p.header = header;
    const int grid = std::min(sms, kMaxCtas);
    switch (columns_for(a.N * a.G)) {
        case 16: return launch<16>(p, grid, stream);
        case 32: return launch<32>(p, grid, stream);
        case 48: return launch<48>(p, grid, stream);
        default: return launch<kWideQ>(p, grid, stream);
    }
}

}  // namespace mcsd
