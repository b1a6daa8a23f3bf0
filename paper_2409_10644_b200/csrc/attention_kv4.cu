// Tree attention (Section 2.2 of the paper) over a prefix cache held in 4 bits (page layout in kv4.cuh), on the
// fifth-generation tensor cores of sm_100a: bf16 tree tensors, head_dim 128, 1 to 96 query columns per work item.
//
// The products are set up transposed, the small dimension (query columns) as the MMA N:
//     S^T[key][query] = K Q^T,     O^T[channel][query] += V^T P^T
// and the A operands live in tensor memory, not in shared memory: thread r of the key warps owns key row r of a
// 128-key tile, thread d of the value warps channel d, and both turn 16-byte pieces of a page (neighbouring threads read
// neighbouring pieces) into operand columns with a shift and a mask per two values and store them with tcgen05.st.
//   * Keys stay codes: 16 + code is exact in bf16, so S' = sum (16 + code) q is exact up to fp32 sums, and the row's scale
//     and offset are applied to the score, where the softmax thread owns the same key row:
//         score = scale_k S' + offset_k (sum of q).
//   * Values become scale_v (16 + code) + offset_v, one packed fused multiply-add per two values, rounded to bf16.
// The rows of the tree itself are read as they are: same operand columns, scale 1, offset 0.
//
// What bounds it: 136 bytes per key and head against 512 in bf16 move the floor of a launch down by 3.8; the unpacking
// (about 20 integer and half-precision instructions per eight keys' and eight values' codes) and the exponentials then
// share the issue slots, so the work is spread over specialised warps:
//   warps 0-3   keys     page pieces -> operand columns (two buffers)
//   warps 4-7   values   page pieces -> operand columns
//   warps 8-15  softmax  two groups that split the query columns; epilogue and merge
//   warp 16     copies whole pages (1 to 4 of them, contiguous) into a ring with cp.async.bulk
//   warp 17     issues the MMAs and owns the tensor memory
//   warps 18-19 bring the queries of the next work item and their sums
//
// Work: one block per multiprocessor walks a contiguous range of the (sequence, key/value head, query block, tile) space,
// cut by cost.  A work item that a range boundary cuts is finished by whichever of its blocks comes last (a counter of
// tiles per item and softmax group; nothing waits): it reads all pieces in block order, so the result does not depend
// on who that is.  Every wait is bounded; one that runs out raises a flag in the workspace header.
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "attention_tc_common.cuh"
#include "kv4.cuh"

namespace mcsd {

namespace {

constexpr int kD = 128;
constexpr int kPageBytes = kv4_page_bytes(kD);
constexpr int kStageBytes = 4 * kPageBytes;      // one tile: 128 rows
constexpr int kValueWarp = 4, kSoftWarp = 8, kCopyWarp = 16, kIssueWarp = 17, kQueryWarp = 18;
constexpr int kThreads = 640;
constexpr int kWideQ = 96;                       // query columns of a work item, at most
constexpr int kStages = 7;
// Tensor-memory columns: scores twice, O^T, keys twice, and values twice where all that fits in 512.
template <int QB>
struct Columns {
    static constexpr int wide = (QB + 31) & ~31;
    static constexpr int S = 0, O = 2 * wide, K = 3 * wide, V = K + 128;
    static constexpr int value_buffers = V + 128 <= kTmemCols ? 2 : 1;
    static_assert(V + 64 * value_buffers <= kTmemCols, "tensor memory");
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
    int* counters;        // [work items][2] tiles that have been finished; zero between launches
    WorkspaceHeader* header;
};

// Per-sequence tables, the same in every block.
struct Plan {
    long long tiles[kMaxBatchTc + 1], cost[kMaxBatchTc + 1];   // of the sequences before b
    int items[kMaxBatchTc + 1];
    int len[kMaxBatchTc], nodes[kMaxBatchTc];
    long long range[2];
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
    const long long r = t - pl.tiles[lo];
    const int it = (int)(r / sh.T);
    s.lt = (int)(r - (long long)it * sh.T);
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

// The block that owns a tile: the inverse of first_tile.
template <int QB>
__device__ __forceinline__ int block_of(const Plan& pl, const Params& p, int b, long long tile_in_b) {
    const Shape sh = shape_of<QB>(pl.len[b], pl.nodes[b], p.G);
    const int w = tile_cost(sh.per_q);
    const long long it = tile_in_b / sh.T, lt = tile_in_b - it * sh.T;
    const long long x = pl.cost[b] + it * ((long long)sh.T * w + kItemCost) + lt * w;
    return (int)(x * pl.blocks / pl.cost[p.B]);
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
        __syncwarp();
        if (tid < 2 && all > 0) pl.range[tid] = first_tile<QB>(pl, p, blockIdx.x + tid);
        if (tid < 2 && all == 0) pl.range[tid] = 0;
    }
    __syncthreads();
}

template <int QB>
struct Small {
    unsigned long long full[kStages], empty[kStages];
    unsigned long long k_full[2], s_full[2], v_full[2], pv_done[2], q_full[2], piece_done[2];
    unsigned long long p_full, drain;
    uint32_t tmem_base;
    int abort_flag;
    int merge[2];                                     // tiles of the item finished before this block's, by group
    alignas(16) float2 kab[4][kTile];                 // scale and offset of a tile's key rows, in score units
    alignas(16) float q_sum[2][QB];
    alignas(16) float ref[2][QB / 2 + 8];             // running reference of a group's own columns
    alignas(16) float alpha[2][QB / 2 + 8];
    alignas(16) float red[2][4][QB / 2 + 8];
    alignas(16) uint64_t anc[MCSD_MAX_NODES * MCSD_MAX_WORDS];
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
// tcgen05.mma with the A operand in tensor memory; see tc_mma_elect for the elected lane
__device__ __forceinline__ void tc_mma_ta_elect(uint32_t d_tmem, uint32_t a_tmem, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
// sixteen consecutive columns of this thread's lane
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
// codes (2i, 2i + 1) of a word as two bf16 numbers 16 + code
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i) {
    const uint32_t x = i == 0 ? w << 3 : w >> (4 * i - 3);
    return (x & 0x00780078u) | 0x41804180u;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// lo += low half, hi += high half of a bf16 pair, in fp32
__device__ __forceinline__ void add_pair(float& lo, float& hi, uint32_t v) {
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %2; add.f32.bf16 %0, a, %0; add.f32.bf16 %1, b, %1;}" : "+f"(lo), "+f"(hi) : "r"(v));
}

template <int QB>
__global__ void __launch_bounds__(kThreads, 1)
tree_attention_kv4_kernel(const Params p) {
    constexpr int CPT = QB / 16;                      // 8-column groups of a softmax thread, at most
    using Col = Columns<QB>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* q_buf = smem;                      // two buffers of QB rows: [2 slabs of 64 channels][QB rows][128 bytes], swizzled
    unsigned char* p_buf = q_buf + 2 * QB * 256;      // P^T: [QB / 8][128 keys][16 bytes]
    unsigned char* ring = p_buf + QB * 256;
    Small<QB>* sm = reinterpret_cast<Small<QB>*>(ring + kStages * kStageBytes);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- set-up; what comes before the wait touches no global memory and overlaps the tail of the preceding kernel
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&sm->full[i], 1); mbar_init(&sm->empty[i], 8); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm->k_full[i], 4);
            mbar_init(&sm->s_full[i], 1);
            mbar_init(&sm->v_full[i], 4);
            mbar_init(&sm->pv_done[i], 1);
            mbar_init(&sm->q_full[i], 2);
            mbar_init(&sm->piece_done[i], 8);
        }
        mbar_init(&sm->p_full, 8);
        mbar_init(&sm->drain, 1);
        sm->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = tid; i < p.N * p.words; i += kThreads) sm->anc[i] = p.anc[i];
    make_plan<QB>(sm->plan, p);
    const Plan& pl = sm->plan;
    const long long t_begin = pl.range[0], t_end = pl.range[1];
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
        constexpr uint32_t q_slab = (QB * 128) >> 4, q_next = (QB * 256) >> 4;
        const uint32_t n_tiles = (uint32_t)(t_end - t_begin);
        Piece s, o;                                   // of the scores and of the products
        long long ts = t_begin, to = t_begin;
        int si = 0, oi = 0;
        uint32_t seg = 0;
        piece_at<QB>(pl, p, ts, t_end, s);
        o = s;
        bool ok = mbar_wait(&sm->q_full[0], 0, abort_flag, hdr, 32);
        for (uint32_t g = 0; g <= n_tiles && ok; ++g) {
            if (g < n_tiles) {
                if (si == s.cnt) {
                    ts += s.cnt;
                    piece_at<QB>(pl, p, ts, t_end, s);
                    si = 0;
                    ++seg;
                    ok = mbar_wait(&sm->q_full[seg & 1u], (seg >> 1) & 1u, abort_flag, hdr, 32);
                    if (!ok) break;
                }
                const uint32_t buf = g & 1u;
                ok = mbar_wait(&sm->k_full[buf], (g >> 1) & 1u, abort_flag, hdr, 33);
                if (!ok) break;
                tc_fence_after();
                const uint32_t idesc = instr_desc((s.Nq + 15) & ~15, 0, 0);
                const uint64_t dq = dq0 + (seg & 1u) * q_next;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    tc_mma_ta_elect(tmem + Col::S + buf * Col::wide, tmem + Col::K + buf * 64 + 8 * k,
                                    dq + (uint32_t)(k >> 2) * q_slab + (uint32_t)(k & 3) * 2u, idesc, k > 0);
                tc_commit_elect(&sm->s_full[buf]);
                ++si;
            }
            if (g >= 1) {
                const uint32_t h = g - 1u;
                if (oi == o.cnt) {
                    to += o.cnt;
                    piece_at<QB>(pl, p, to, t_end, o);
                    oi = 0;
                }
                ok = mbar_wait(&sm->v_full[h & 1u], (h >> 1) & 1u, abort_flag, hdr, 34);
                if (!ok) break;
                ok = mbar_wait(&sm->p_full, h & 1u, abort_flag, hdr, 35);
                if (!ok) break;
                tc_fence_after();
                const uint32_t idesc = instr_desc((o.Nq + 15) & ~15, 0, 1);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    tc_mma_ta_elect(tmem + Col::O, tmem + Col::V + (Col::value_buffers == 2 ? (h & 1u) * 64 : 0u) + 8 * k, dp0 + (uint32_t)(k * (256 >> 4)), idesc, (oi > 0) | (k > 0));
                tc_commit_elect(&sm->pv_done[h & 1u]);
                ++oi;
            }
        }
        tc_commit_elect(&sm->drain);                  // all MMAs have finished before tensor memory is released
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
                    v = *reinterpret_cast<const uint4*>(p.q + (((size_t)s.b * p.Hkv * p.G + h) * p.N + n) * kD + c * 8);
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
        const int r = tid;
        const uint32_t lane_addr = tmem + ((uint32_t)(warp * 32) << 16);
        uint32_t g = 0, f = 0;
        bool ok = true;
        for (long long t = t_begin; t < t_end && ok;) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            for (int i = s.lt; i < s.lt + s.cnt && ok; ++i, ++g) {
                const uint32_t buf = g & 1u, dst = lane_addr + Col::K + buf * 64;
                if (i < s.Tp) {
                    const uint32_t st = f % kStages;
                    ok = mbar_wait(&sm->full[st], (f / kStages) & 1u, abort_flag, hdr, 37);
                    if (!ok) break;
                    const unsigned char* page = ring + st * kStageBytes + warp * kPageBytes;   // rows 32 warp .. of the tile
                    uint4 x[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[c] = *reinterpret_cast<const uint4*>(page + c * (kPageRows * 16) + lane * 16);
                    const unsigned short* sc = reinterpret_cast<const unsigned short*>(page + kv4_scales_at(kD));
                    const float a = bf16_bits_to_f32(sc[lane]), b = bf16_bits_to_f32(sc[kPageRows + lane]);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->empty[st]);
                    ++f;
                    // The buffer is free once the scores of the tile before last are done.  They were issued after the
                    // softmax warps had finished tile g - 4, whose scales the entry below held.
                    if (g >= 2) ok = mbar_wait(&sm->s_full[buf], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 38);
                    if (!ok) break;
                    tc_fence_after();
                    sm->kab[g & 3u][r] = make_float2(a * p.scale_log2, b * p.scale_log2);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
                        uint32_t y[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = code_pair(w[e >> 2], e & 3);
                        tc_st16(dst + 16 * c, y);
                    }
                } else {
                    const int n = (i - s.Tp) * kTile + r;
                    if (g >= 2) ok = mbar_wait(&sm->s_full[buf], ((g - 2u) >> 1) & 1u, abort_flag, hdr, 38);
                    if (!ok) break;
                    tc_fence_after();
                    sm->kab[g & 3u][r] = make_float2(p.scale_log2, 0.f);
                    const uint4* row = reinterpret_cast<const uint4*>(p.k_tree + (((size_t)s.b * p.Hkv + s.hk) * p.N + n) * kD);
#pragma unroll
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
        bool ok = true;
        for (long long t = t_begin; t < t_end && ok;) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            for (int i = s.lt; i < s.lt + s.cnt && ok; ++i, ++g) {
                const uint32_t dst = lane_addr + (NV == 2 ? (g & 1u) * 64 : 0u);
                const uint32_t st = f % kStages;
                if (i < s.Tp) ok = mbar_wait(&sm->full[st], (f / kStages) & 1u, abort_flag, hdr, 39);
                // the buffer is free once the products of the tile that used it are done
                if (ok && g >= NV) ok = mbar_wait(&sm->pv_done[(g - NV) & 1u], ((g - NV) >> 1) & 1u, abort_flag, hdr, 40);
                if (!ok) break;
                tc_fence_after();
                if (i < s.Tp) {
                    const int valid = min(kTile, s.L - i * kTile);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const unsigned char* page = ring + st * kStageBytes + c * kPageBytes;
                        const uint4 x = *reinterpret_cast<const uint4*>(page + kv4_values_at(kD) + d * 16);
                        const uint4* sc = reinterpret_cast<const uint4*>(page + kv4_scales_at(kD) + 4 * kPageRows);   // scales, then offsets
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                        uint32_t y[16];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint4 a = sc[j], b = sc[4 + j];
                            y[4 * j] = fma_bf16x2(code_pair(w[j], 0), a.x, b.x);
                            y[4 * j + 1] = fma_bf16x2(code_pair(w[j], 1), a.y, b.y);
                            y[4 * j + 2] = fma_bf16x2(code_pair(w[j], 2), a.z, b.z);
                            y[4 * j + 3] = fma_bf16x2(code_pair(w[j], 3), a.w, b.w);
                        }
                        // rows past the end of the prefix have probability zero, but may hold anything: 0 * NaN would be NaN
                        if (valid < kTile) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const int n = 32 * c + 2 * e;
                                y[e] &= (n < valid ? 0xFFFFu : 0u) | (n + 1 < valid ? 0xFFFF0000u : 0u);
                            }
                        }
                        tc_st16(dst + 16 * c, y);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->empty[st]);
                    ++f;
                } else {
                    const int n0 = (i - s.Tp) * kTile, n1 = min(kTile, s.Nb - n0);
                    const unsigned short* col = reinterpret_cast<const unsigned short*>(p.v_tree) + (((size_t)s.b * p.Hkv + s.hk) * p.N + n0) * kD + d;
#pragma unroll
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
        // ---- softmax, epilogue, merge: group wg has about half of the query columns, thread r key row r
        const int wg = (warp - kSoftWarp) >> 2, wq = warp & 3, r = tid & 127;
        const int bar_id = 1 + wg;
        const uint32_t lane_addr = tmem + ((uint32_t)(wq * 32) << 16);
        float* const ref = sm->ref[wg];
        float* const alph = sm->alpha[wg];
        uint32_t g = 0, seg = 0;
        bool failed = false;
        for (long long t = t_begin; t < t_end; ++seg) {
            Piece s;
            piece_at<QB>(pl, p, t, t_end, s);
            const int n8 = (s.Nq + 7) >> 3;
            const int g0 = wg ? (n8 + 1) / 2 : 0;                // first 8-column group of this group, and how many
            const int ncg = wg ? n8 / 2 : (n8 + 1) / 2;
            const int col0 = 8 * g0;
            const float* qs = &sm->q_sum[seg & 1u][col0];
            float lsum[CPT][8];
#pragma unroll
            for (int j = 0; j < CPT; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) lsum[j][k] = 0.f;
            if (r < 8 * ncg) ref[r] = -1e30f;                    // below any score: the first tile sets it
            if (group_sync_any(bar_id, failed)) { failed = true; break; }

            for (int i = s.lt; i < s.lt + s.cnt; ++i, ++g) {
                const uint32_t buf = g & 1u;
                const bool tree = i >= s.Tp;
                const int row = (tree ? i - s.Tp : i) * kTile + r;
                const bool plain = !tree && (i + 1) * kTile <= s.L;   // every key there and visible to every query
                unsigned long long cm = 0;                        // columns that see this thread's key
                if (!plain) {
                    const int nq = min(s.Nq - col0, 8 * ncg);
                    if (!tree) {
                        if (row < s.L) cm = (1ull << max(nq, 0)) - 1ull;
                    } else if (row < s.Nb) {
                        int n = (s.q0 + col0) / p.G, rest = (s.q0 + col0) - n * p.G;
                        for (int c = 0; c < nq; ++c) {
                            cm |= (unsigned long long)((sm->anc[n * p.words + (row >> 6)] >> (row & 63)) & 1ull) << c;
                            if (++rest == p.G) { rest = 0; ++n; }
                        }
                    }
                }
                if (!mbar_wait(&sm->s_full[buf], (g >> 1) & 1u, abort_flag, hdr, 41)) failed = true;
                tc_fence_after();
                const uint32_t s_addr = lane_addr + Col::S + buf * Col::wide + col0;
                const float2 ab = sm->kab[g & 3u][r];
                uint32_t pk[CPT][4];
                float dmax = -INFINITY;
                auto sweep = [&](auto masked_tag) {
                    constexpr bool MASKED = decltype(masked_tag)::value;
                    dmax = -INFINITY;
#pragma unroll
                    for (int j = 0; j < CPT; ++j) {
                        if (j < ncg) {
                            float y[8];
                            tc_ld8(s_addr + 8 * j, y);
                            const float4 q0 = *reinterpret_cast<const float4*>(qs + 8 * j), q1 = *reinterpret_cast<const float4*>(qs + 8 * j + 4);
                            const float4 m0 = *reinterpret_cast<const float4*>(ref + 8 * j), m1 = *reinterpret_cast<const float4*>(ref + 8 * j + 4);
                            const float qv[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
                            const float mv[8] = {m0.x, m0.y, m0.z, m0.w, m1.x, m1.y, m1.z, m1.w};
                            tc_wait_ld();
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                y[k] = fmaf(y[k], ab.x, fmaf(qv[k], ab.y, -mv[k]));
                                if (MASKED) y[k] = ((cm >> (8 * j + k)) & 1ull) ? y[k] : -INFINITY;
                            }
                            dmax = fmaxf(dmax, fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7]))));
#pragma unroll
                            for (int k = 0; k < 8; k += 2) {
                                const __nv_bfloat162 h = __floats2bfloat162_rn(ex2_approx(y[k]), ex2_approx(y[k + 1]));
                                pk[j][k >> 1] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                        }
                    }
                };
                if (plain) sweep(std::false_type{}); else sweep(std::true_type{});
                // one vote per group: does any score exceed its reference by more than the lazy threshold?
                if (group_sync_any(bar_id, dmax > kLazyTau || failed)) {
                    if (group_sync_any(bar_id, failed)) { failed = true; break; }
                    // exact column maxima of the tile, new references, what was accumulated rescaled
#pragma unroll
                    for (int j = 0; j < CPT; ++j) {
                        if (j < ncg) {
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
                    }
                    group_sync_any(bar_id, false);
                    bool need = false;
                    if (r < 8 * ncg) {
                        const float top = fmaxf(fmaxf(sm->red[wg][0][r], sm->red[wg][1][r]), fmaxf(sm->red[wg][2][r], sm->red[wg][3][r]));
                        const float old = ref[r];
                        float a = 1.f;
                        if (top > old) {
                            a = exp2f(old - top);
                            ref[r] = top;
                            need = i > s.lt;
                        }
                        alph[r] = a;
                    }
                    const bool rescale = group_sync_any(bar_id, need);
                    if (rescale) {
                        if (g > 0 && !mbar_wait(&sm->pv_done[(g - 1u) & 1u], ((g - 1u) >> 1) & 1u, abort_flag, hdr, 42)) failed = true;
                        tc_fence_after();
#pragma unroll
                        for (int j = 0; j < CPT; ++j) {
                            if (j < ncg) {
                                float o[8];
                                tc_ld8(lane_addr + Col::O + col0 + 8 * j, o);
                                tc_wait_ld();
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    o[k] *= alph[8 * j + k];
                                    lsum[j][k] *= alph[8 * j + k];
                                }
                                tc_st8(lane_addr + Col::O + col0 + 8 * j, o);
                            }
                        }
                        tc_wait_st();
                    }
                    if (plain) sweep(std::false_type{}); else sweep(std::true_type{});
                }
                // row sums of the rounded weights, then P^T once the products of the previous tile no longer read it
#pragma unroll
                for (int j = 0; j < CPT; ++j)
                    if (j < ncg) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) add_pair(lsum[j][2 * k], lsum[j][2 * k + 1], pk[j][k]);
                    }
                if (g > 0 && !mbar_wait(&sm->pv_done[(g - 1u) & 1u], ((g - 1u) >> 1) & 1u, abort_flag, hdr, 43)) failed = true;
#pragma unroll
                for (int j = 0; j < CPT; ++j)
                    if (j < ncg)
                        *reinterpret_cast<uint4*>(p_buf + (g0 + j) * 2048 + r * 16) = make_uint4(pk[j][0], pk[j][1], pk[j][2], pk[j][3]);
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm->p_full);
            }
            if (group_sync_any(bar_id, failed)) { failed = true; break; }

            // ---- the piece is done: row sums over the 128 key rows, eight columns at a time.  Exchanging halves leaves
            // lane x with the sum over the warp of column (x >> 2) & 7 (bits 4, 3, 2 of the lane, in this order).
#pragma unroll
            for (int j = 0; j < CPT; ++j) {
                if (j < ncg) {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = lsum[j][k];
#pragma unroll
                    for (int half = 4, bit = 16; half > 0; half >>= 1, bit >>= 1) {
                        const bool up = lane & bit;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if (k < half) {
                                const float got = __shfl_xor_sync(0xffffffffu, up ? v[k] : v[k + half], bit);
                                v[k] = (up ? v[k + half] : v[k]) + got;
                            }
                        }
                    }
                    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
                    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);
                    if ((lane & 3) == 0) sm->red[wg][wq][8 * j + ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1)] = v[0];
                }
            }
            if (!mbar_wait(&sm->pv_done[(g - 1u) & 1u], ((g - 1u) >> 1) & 1u, abort_flag, hdr, 44)) failed = true;
            tc_fence_after();
            if (group_sync_any(bar_id, failed)) { failed = true; break; }
            const bool whole = s.cnt == s.T;
            const int slot = 2 * (int)blockIdx.x + (t > t_begin ? 1 : 0);
            if (r < 8 * ncg) {
                const float l = (sm->red[wg][0][r] + sm->red[wg][1][r]) + (sm->red[wg][2][r] + sm->red[wg][3][r]);
                if (whole) {
                    alph[r] = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
                } else if (col0 + r < s.Nq) {
                    p.part_ml[((size_t)slot * 2 + 0) * kWideQ + col0 + r] = ref[r];
                    p.part_ml[((size_t)slot * 2 + 1) * kWideQ + col0 + r] = l;
                }
            }
            group_sync_any(bar_id, false);
            // rows of `out` of the group's columns: query j = q0 + column is head j % G, node j / G
            auto put = [&](int c, float v) {
                const int j = s.q0 + c, n = j / p.G, h = s.hk * p.G + (j - n * p.G);
                p.out[(((size_t)s.b * p.Hkv * p.G + h) * p.N + n) * kD + r] = __float2bfloat16_rn(v);
            };
#pragma unroll
            for (int j = 0; j < CPT; ++j) {
                if (j < ncg) {
                    float o[8];
                    tc_ld8(lane_addr + Col::O + col0 + 8 * j, o);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int c = col0 + 8 * j + k;
                        if (c < s.Nq) {
                            if (whole) put(c, o[k] * alph[8 * j + k]);
                            else p.part_o[((size_t)slot * kWideQ + c) * kD + r] = o[k];
                        }
                    }
                }
            }
            if (!whole) {
                // the group that finishes an item's last tile merges its columns of all pieces
                __threadfence();
                group_sync_any(bar_id, false);
                if (r == 0) sm->merge[wg] = atomicAdd(&p.counters[2 * s.item + wg], s.cnt);
                group_sync_any(bar_id, false);
                if (sm->merge[wg] + s.cnt == s.T) {
                    __threadfence();
                    const long long it0 = (long long)(s.item - pl.items[s.b]) * s.T;     // the item's first tile, in its sequence
                    const int c0 = block_of<QB>(pl, p, s.b, it0), c1 = block_of<QB>(pl, p, s.b, it0 + s.T - 1);
                    const long long first = pl.tiles[s.b] + it0;
                    // slot of block c's piece of this item, or -1
                    auto slot_of = [&](int c) -> int {
                        const long long a = first_tile<QB>(pl, p, c), b = first_tile<QB>(pl, p, c + 1);
                        if (max(a, first) >= min(b, first + s.T)) return -1;
                        return 2 * c + (a < first ? 1 : 0);
                    };
                    if (r < 8 * ncg && col0 + r < s.Nq) {
                        float M = -INFINITY, l = 0.f;
                        for (int c = c0; c <= c1; ++c) {
                            const int sl = slot_of(c);
                            if (sl >= 0) M = fmaxf(M, __ldcg(&p.part_ml[((size_t)sl * 2) * kWideQ + col0 + r]));
                        }
                        for (int c = c0; c <= c1; ++c) {
                            const int sl = slot_of(c);
                            if (sl >= 0)
                                l += exp2f(__ldcg(&p.part_ml[((size_t)sl * 2) * kWideQ + col0 + r]) - M) *
                                     __ldcg(&p.part_ml[((size_t)sl * 2 + 1) * kWideQ + col0 + r]);
                        }
                        ref[r] = M;
                        alph[r] = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
                    }
                    group_sync_any(bar_id, false);
#pragma unroll 1
                    for (int j = 0; j < ncg; ++j) {
                        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                        for (int c = c0; c <= c1; ++c) {
                            const int sl = slot_of(c);
                            if (sl < 0) continue;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const int q = col0 + 8 * j + k;
                                if (q < s.Nq)
                                    acc[k] = fmaf(exp2f(__ldcg(&p.part_ml[((size_t)sl * 2) * kWideQ + q]) - ref[8 * j + k]),
                                                  __ldcg(&p.part_o[((size_t)sl * kWideQ + q) * kD + r]), acc[k]);
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (col0 + 8 * j + k < s.Nq) put(col0 + 8 * j + k, acc[k] * alph[8 * j + k]);
                    }
                    if (r == 0) p.counters[2 * s.item + wg] = 0;
                    group_sync_any(bar_id, false);               // the references are read by all
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm->piece_done[seg & 1u]);
            t += s.cnt;
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
    return per <= 16 ? 16 : per <= 32 ? 32 : per <= 48 ? 48 : per <= 64 ? 64 : kWideQ;
}

template <int QB>
int launch(const Params& p, int grid, cudaStream_t stream) {
    constexpr size_t smem_bytes = 1024 + 3 * QB * 256 + (size_t)kStages * kStageBytes + sizeof(Small<QB>);
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

bool kv4_tc_shape(int B, int H, int G, int N, int D, int L_max, int dtype) { return tc_shape_supported(B, H, G, N, D, L_max, dtype); }

size_t kv4_tc_workspace_bytes(int B, int H, int G, int N) {
    const size_t blocks_q = ((size_t)G * N + kWideQ - 1) / kWideQ * 2;   // narrower launches cut finer, by less than two
    return kMlBytes + kOBytes + align_up((size_t)B * (H / G) * blocks_q * 2 * sizeof(int), 256);
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
        case 64: return launch<64>(p, grid, stream);
        default: return launch<kWideQ>(p, grid, stream);
    }
}

}  // namespace mcsd
