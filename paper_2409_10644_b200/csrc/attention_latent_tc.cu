// Tree attention over a latent cache on the fifth-generation tensor cores of sm_100a: bf16, rank 512, rotated part 64.
//
//   S = Q K^T,  P = exp2(scale S - ref),  O += P V,   Q: 128 query rows of 576, K: keys of 576, V: their first 512 values
//
// All heads and nodes of a sequence share the keys, so its H * n_active query rows are one matrix; a work item is 128 of
// them.  Their 128 x 512 fp32 accumulators fill the tensor memory of one multiprocessor and leave no room for S, so a pair
// of blocks (a cluster of two) takes an item together: tcgen05.mma.cta_group::2 with M = 128 gives each 64 rows, whose
// accumulators take 256 columns there, rows in lanes 0..63 and the upper half of N in lanes 64..127.  The products of this
// shape run at the full rate with N = 256 (64 cycles each, measured; 50 with N = 128), so a tile has 256 keys: S is 128
// columns, twice, and tensor memory is full.
//
// A block loads its half of what a product needs: for S its half of the keys, 64 channels at a time, for O its half of the
// channels, 64 keys at a time; both are 16 KB, and pass through two rings of four and three slots.  S and O are issued by two
// warps, each from its own ring: four products, the wait for their slot and the commit that releases it take a warp 370 to
// 470 cycles and the tensor cores 256 (measured), so that one warp issuing both would pace them; and S of a tile or item
// runs into O of the last one by itself.  A warp issues convergently through one elected lane, its operands then lie in
// uniform registers (128 cycles a product from a single thread's branch).
//
// A tile always ends at the last key of its range and starts a multiple of 32 keys before: a ragged tile overlaps the tile
// before it (or starts before the first row, where TMA gives zeros) and masks what it has no claim to, so that no row behind a
// sequence's end ever meets a product.
//
// Weights are rounded to bf16, since both operands of a product are of one type and the values are bf16: half a step, 2^-8 of each.
// Their sum is taken before that, in fp32.  Against 64 bits the outputs of 45-node trees are off by 2.0e-3 of their size, where one
// rounding of exact outputs leaves 1.7e-3.
//
// The launch's tiles are numbered (sequence, row block, tile) and cut into equal ranges, one a pair; where a cut falls
// inside an item, the pieces write unnormalised rows and count themselves in.  An item of two or three pieces is joined by the
// pair that starts it, from tensor memory: the others wrote theirs early, as the first of their ranges (with three instead of
// two 32 single tokens of 128 heads over 4000 keys take 42 instead of 56 us).  Where there are more, the pairs wait at the end of
// their ranges and join a share of its channels each (only as many pairs get work as keeps items in three pieces, where that is
// sooner done).  Both bring what they join into shared memory at once: the range is over, its memory free.
//
// All blocks usually run at a time, one a multiprocessor; where others hold multiprocessors (a kernel of another stream), a pair
// must not wait for one that cannot start before it leaves.  So it waits for a millisecond at most, then notes that it is gone,
// and the pair that brings the last piece joins the shares of those that are: no result depends on which blocks run together.  (How
// long it waits is a parameter of the launch, which tests set to nothing and to a few thousand cycles.)
//
// What bounds it.  Many rows: the tensor cores; 128 heads of a 74-node tree over 32768 keys run at 1.59 PFLOP/s, the rate of a
// plain matrix product on this card.  A tile takes 3.3 us, an item 4 more for its last products and its output, which nothing
// covers, and a launch 9 to start: 16 trees of 45 nodes and 32 heads over 4096 keys 180 us, 1.15 PFLOP/s.  One row block a
// sequence: memory, at 7 TB/s once it streams; 8 tokens of 128 heads over up to 32001 keys 59 us, of which 20 are start and
// joining.  One token over 1001 keys: 18 us of latencies (5 until the first scores, 5 for two tiles, 7 to join).
//
// The five roles run side by side, each its own loop: unrolled, they did not fit the instruction caches, and a tile took 4.9 us
// instead of 3.4 (the loops of S over nine chunks and of O over four quarters are rolled for that alone).
//
// Warps of a block: 0 loads for S, 1 issues it, 2 loads for O, 3 issues it (1 and 3 in the first block of the pair), 4 to 11
// fetch queries, do the softmax and the output.  Every wait is bounded; one that runs out raises a flag in the workspace header,
// all roles drain and the blocks exit.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <mutex>

#include "attention_tc_common.cuh"
#include "f32x2.cuh"
#include "latent.cuh"

namespace mcsd {

constexpr int kLtRank = 512, kLtRot = 64, kLtWidth = kLtRank + kLtRot;
constexpr int kLtChunks = kLtWidth / 64;             // 64-channel chunks of a row
constexpr int kLtThreads = 384;
constexpr int kLtTile = 256;                         // keys of a tile
constexpr int kLtKeySlots = 4, kLtValueSlots = 3, kLtSlots = kLtKeySlots + kLtValueSlots, kLtSlotBytes = 16384;
constexpr int kLtQBytes = kLtChunks * 8192, kLtPBytes = 4 * 8192;      // queries, weights of a tile
constexpr int kLtMaxBatch = 256;
constexpr int kLtMaxPairs = kTcMaxBlocks / 2;
constexpr int kLtFew = 3;                            // pieces of an item that are joined by the pair that starts it
constexpr int kLtGone = 1 << 8, kLtLeft = 1 << 16;   // an item's counter: pieces that are in, pairs that wait no more, pairs done with it
constexpr int kLtGoneWords = kCountersPerBlock - 1;  // and the pairs that wait no more, a bit each
static_assert(kLtMaxPairs <= 32 * kLtGoneWords && kLtMaxPairs < 256, "an item's counters");
constexpr long long kLtPatience = 1 << 21;           // cycles, about a millisecond
constexpr int kLtColO = 0, kLtColS = 256;            // tensor memory: O 256 columns, S 128 twice

struct LtParams {
    LatentArgs a;
    float scale_log2;
    float* part_o;                                   // unnormalised rows of pieces, two slots a pair (see lt_part)
    float2* part_ml;                                 // [2 * pairs][128]  reference (log2), sum
    int* counters;                                   // [2 * pairs][kCountersPerBlock] of the item that a block starts
    WorkspaceHeader* header;
    long long patience;                              // cycles that a pair waits for pieces of others
};
struct LtMaps {
    CUtensorMap m[8];                                // boxes of 16, 32, 64, 128 rows: cache, then tree
};

struct LtItem {
    int b, rb, L, Nb, nP, nt;      // sequence, row block; prefix length, nodes; prefix tiles, tiles
    int t0, t1;                    // this pair's tiles
    int unit0;                     // the item's first unit
    __device__ __forceinline__ void uniform() {      // alike in all lanes: say so
        L = __shfl_sync(0xffffffffu, L, 0);
        Nb = __shfl_sync(0xffffffffu, Nb, 0);
        nP = __shfl_sync(0xffffffffu, nP, 0);
        t0 = __shfl_sync(0xffffffffu, t0, 0);
        t1 = __shfl_sync(0xffffffffu, t1, 0);
    }
};
struct LtSmall {
    unsigned long long full[kLtSlots], empty[kLtSlots];          // slots of S, then of O
    unsigned long long s_full[2], s_free[2], p_full[4], p_free[4], pv_done, q_full;
    uint32_t tmem_base;
    int abort_flag;
    int pairs;                                       // pairs with work
    int joins;                                       // items to join at the end of the range (the first and the last at most)
    LtItem join[2];
    int join_in[2];                                  // their counter as this pair's piece found it
    int all_in;                                      // what a wait for pieces found
    uint32_t shares[kLtGoneWords];                   // shares of an item that this pair joins
    int total;                                       // units of the launch
    int items;                                       // work items of the launch
    int scan[kLtThreads / 32];
    int cum[kLtMaxBatch + 1];                        // units before a sequence
    float red[2][4][64];                             // row maxima of a tile's quarters, by tile parity
    float lsum[4][64];
};
constexpr int kLtSmem = 1024 + kLtQBytes + kLtPBytes + kLtSlots * kLtSlotBytes + (int)sizeof(LtSmall);
static_assert((kLtFew - 1) * 8 * 4096 <= kLtQBytes && kLtQBytes <= kLtSlots * kLtSlotBytes, "a quarter of the pieces that are joined at the start");
static_assert(kLtSmem <= kSmemLimit, "a block's shared memory");

// ------------------------------------------------------------------ PTX of a pair of blocks
__device__ __forceinline__ uint32_t leader_addr(uint32_t addr) {      // the same shared variable in the pair's first block
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
// Arrival at a barrier of the pair's first block.  What is handed over with it lies in this block's own shared or tensor memory
// and is read by products alone: the writer has made it visible to them before (fence.proxy.async, tcgen05.fence), so the
// arrival needs no release at cluster scope, which costs a memory barrier (1300 cycles a tile, measured).
__device__ __forceinline__ void arrive_pair(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// Both by a warp that is together, through the lane for which `one` is not 0 (the same lane for both).
__device__ __forceinline__ uint32_t elect_lane() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e;
}
__device__ __forceinline__ void pair_mma(uint32_t one, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 e, %5, 0;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(one) : "memory");
}
__device__ __forceinline__ void pair_commit(uint32_t one, void* bar) {              // the barrier of both blocks
    const uint16_t both = 3;
    asm volatile("{\n\t.reg .pred e;\n\t"
                 "setp.ne.b32 e, %2, 0;\n\t"
                 "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
                 ::"r"(smem_u32(bar)), "h"(both), "r"(one) : "memory");
}
__device__ __forceinline__ void cluster_sync_all() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Lanes come here from waits of one thread and from loops of different trips (rows behind the last one join nothing).
__device__ __forceinline__ void softmax_sync() {
    __syncwarp();
    asm volatile("bar.sync 1, 256;" ::: "memory");
}
// 32 consecutive fp32 columns of this thread's lane; the caller waits with tc_wait_ld()
__device__ __forceinline__ void tc_ld32(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}

// ------------------------------------------------------------------ the cut of a launch
// Cost of an item's parts in units of 525 cycles (a least-squares fit of when pairs finished, over launches of few and many, long
// and short items): a tile has a fixed part (its waits) and one by its keys (its products), an item starts with its queries and
// ends with its output.  A pair takes the tiles that start in its range of the launch's units.
constexpr int kLtItemCost = 14, kLtJoinCost = 25;      // the latter: an item in more than kLtFew pieces
__host__ __device__ __forceinline__ int lt_tile_cost(int keys) { return 6 + (4 * keys + 255) / 256; }
__host__ __device__ __forceinline__ int lt_row_blocks(int H, int Nb) { return (H * Nb + 127) / 128; }
__device__ __forceinline__ int lt_len(const LatentArgs& a, int b) { return min(max(a.seq_lens[b], 0), a.L_max); }
__device__ __forceinline__ int lt_nodes(const LatentArgs& a, int b) { return a.n_active ? min(max(a.n_active[b], 0), a.N) : a.N; }

// The tiles of an item: full prefix tiles, a shorter one, full tree tiles, a shorter one.
struct LtShape {
    static constexpr int cost = 10;                            // of a full tile
    int full, rest_cost, tree_full, tree_rest_cost;
    __host__ __device__ __forceinline__ LtShape(int L, int Nb) {
        const int rest = L % kLtTile, tree_rest = Nb % kLtTile;
        full = L / kLtTile;
        rest_cost = rest ? lt_tile_cost(rest) : 0;
        tree_full = Nb / kLtTile;
        tree_rest_cost = tree_rest ? lt_tile_cost(tree_rest) : 0;
    }
    __host__ __device__ __forceinline__ int prefix_tiles() const { return full + (rest_cost > 0); }
    __host__ __device__ __forceinline__ int tiles() const { return prefix_tiles() + tree_full + (tree_rest_cost > 0); }
    __host__ __device__ __forceinline__ int total() const { return kLtItemCost + full * cost + rest_cost + tree_full * cost + tree_rest_cost; }
    // where tile t starts, in units from the item's start
    __host__ __device__ __forceinline__ int start(int t) const {
        return kLtItemCost + (t <= full ? t * cost : full * cost + rest_cost + (t - prefix_tiles()) * cost);
    }
    // the first tile that starts at x or later (tiles() where there is none)
    __host__ __device__ __forceinline__ int tile_from(int x) const {
        const int y = x - kLtItemCost, z = y - full * cost;
        if (y <= 0) return 0;
        if (z <= 0) return (y + cost - 1) / cost;
        const int after = z - rest_cost;                       // past the shorter prefix tile
        const int t = prefix_tiles() + (after > 0 ? (after + cost - 1) / cost : 0);
        return t < tiles() ? t : tiles();
    }
};
// first unit of pair c
__device__ __forceinline__ int lt_first(int c, int total, int pairs) { return (int)((long long)c * total / pairs); }
__device__ __forceinline__ int lt_pair_of(int unit, int total, int pairs) { return (int)((((long long)unit + 1) * pairs - 1) / total); }

// Walks the items of a pair's range; every role of both blocks walks alike.
struct LtWalk {
    int u, end, b;
    __device__ __forceinline__ void start(const LtSmall* sm, int pair) {
        b = 0;
        u = end = 0;
        if (pair < sm->pairs) {
            u = lt_first(pair, sm->total, sm->pairs);
            end = lt_first(pair + 1, sm->total, sm->pairs);
        }
    }
    __device__ __forceinline__ bool next(const LtSmall* sm, const LatentArgs& a, LtItem& it) {
        while (u < end) {
            while (sm->cum[b + 1] <= u) ++b;
            it.b = b;
            it.L = lt_len(a, b);
            it.Nb = lt_nodes(a, b);
            const LtShape x(it.L, it.Nb);
            it.nP = x.prefix_tiles();
            it.nt = x.tiles();
            const int off = u - sm->cum[b], total = x.total();
            it.rb = off / total;
            const int rem = off - it.rb * total;
            it.unit0 = u - rem;
            const int stop = min(end, it.unit0 + total);
            it.t0 = x.tile_from(rem);
            it.t1 = x.tile_from(stop - it.unit0);
            u = stop;
            if (it.t1 > it.t0) return true;
        }
        return false;
    }
};
// The pairs that have tiles of an item: a range of units is no shorter than a tile, so that none between them is without.
__device__ __forceinline__ void lt_owners(const LtSmall* sm, const LtItem& it, int& first, int& last) {
    const LtShape x(it.L, it.Nb);
    first = lt_pair_of(it.unit0 + x.start(0), sm->total, sm->pairs);
    last = lt_pair_of(it.unit0 + x.start(it.nt - 1), sm->total, sm->pairs);
}
struct LtTile {
    int lo, start, kpc;            // first key it has a claim to, first key that is loaded, keys of a block (16 .. 128)
    bool tree;
};
__device__ __forceinline__ LtTile lt_tile(const LtItem& it, int t) {
    LtTile x;
    x.tree = t >= it.nP;
    x.lo = (x.tree ? t - it.nP : t) * kLtTile;
    const int stop = min(x.lo + kLtTile, x.tree ? it.Nb : it.L);
    x.kpc = (stop - x.lo + 31) / 32 * 16;
    x.start = stop - 2 * x.kpc;
    return x;
}

// A tile's keys in quarters: up to 64 keys of the first block's half, the rest of that half, and the same of the second's.
// Quarters pass from the softmax to the products one by one, so that weights are written while the products of the tile
// before still read theirs.
__device__ __forceinline__ int lt_quarter(int kpc, int q) { return min(max(kpc - 64 * (q & 1), 0), 64); }
__device__ __forceinline__ int lt_quarter_start(int kpc, int q) { return (q >> 1) * kpc + 64 * (q & 1); }

__device__ __forceinline__ uint64_t anc_word(const uint64_t* w, int words, int i) { return i >= 0 && i < words ? w[i] : 0; }
// 32 bits of a mask row from bit `pos` on (which may lie before the first bit: zeros)
__device__ __forceinline__ uint32_t anc_bits(const uint64_t* w, int words, int pos) {
    const int i = pos >> 6, s = pos & 63;
    uint64_t v = anc_word(w, words, i) >> s;
    if (s) v |= anc_word(w, words, i + 1) << (64 - s);
    return (uint32_t)v;
}

// Pieces lie as tensor memory does, four columns of its 128 lanes (a row and half of the channels each) side by side, so that a
// warp writes and reads 512 bytes at a time: [slot][block of the pair][64 quads of columns][128 lanes][4].
__device__ __forceinline__ float4* lt_part(const LtParams& p, int slot, int rank, int quad, int tlane) {
    return reinterpret_cast<float4*>(p.part_o) + (((long long)slot * 2 + rank) * 64 + quad) * 128 + tlane;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float4 lds16(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float2 lds8(uint32_t at) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
// Waits (one thread) until `count` pieces are in or patience runs out; then this pair is counted as gone, unless they came in
// just before.  Returns whether they are in.  `bit` of `word` goes before the count: who sees the count finds it.
__device__ __noinline__ bool lt_await(LtSmall* sm, long long patience, int* counter, int count, bool ok, int* word, int bit) {
    const long long t0 = clock64();
    while (ok && clock64() - t0 < patience && !*(volatile int*)&sm->abort_flag) {
        int seen;
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
        if ((seen & (kLtGone - 1)) >= count) return true;
    }
    if (bit) atomicOr(word, bit);
    __threadfence();
    const bool in = (atomicAdd(counter, kLtGone) & (kLtGone - 1)) >= count;
    __threadfence();
    return in;
}
// This pair is done with an item in `count` pieces: the last one to leave puts its counters back to zero.
__device__ __forceinline__ void lt_leave(int* counter, int count) {
    if (atomicAdd(counter, kLtLeft) / kLtLeft == count - 1)
        for (int k = 0; k < kCountersPerBlock; ++k) counter[k] = 0;
}
// Share k of `shares` of the columns of an item in `count` pieces, by the 256 threads of the softmax warps: a thread has a lane of tensor memory and
// every other quad of columns.  The range is over, so that all of a block's operand memory is free: the pieces' values come
// there, as many at a time as fit, and are joined in their order.
constexpr int kLtJoinSlots = 44;                                  // of 16 bytes a thread
static_assert((kLtJoinSlots * 256 * 16) + kLtMaxPairs * 512 <= kLtQBytes + kLtPBytes + kLtSlots * kLtSlotBytes, "joining");
__device__ __noinline__ void lt_join_share(const LtParams& p, const LtItem& it, uint32_t smem, int first, int count, int k, int shares, int rank, int tid) {
    const LatentArgs& a = p.a;
    const int tlane = tid & 127, row = tlane & 63, half = tlane >> 6, r = it.rb * 128 + rank * 64 + row;
    const bool in = r < a.H * it.Nb;
    const uint32_t ml = smem + kLtJoinSlots * 4096, own = smem + tid * 16;
    // piece 0 lies in its pair's second slot, the others in the first
    for (int i = tid; i < 32 * count; i += 256) {
        const int piece = i >> 5, slot = 2 * (first + piece) + (piece == 0);
        copy16(ml + piece * 512 + (i & 31) * 16, p.part_ml + slot * 128 + rank * 64 + 2 * (i & 31));
    }
    const int q0 = 64 * k / shares + (tid >> 7), q1 = 64 * (k + 1) / shares, n = in && q1 > q0 ? (q1 - q0 + 1) / 2 * count : 0;
    float top = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    int quad = q0, piece = 0, fq = q0, fp = 0;
    const int h = in ? r / it.Nb : 0, node = in ? r - h * it.Nb : 0;
    __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(a.out) + (((long long)it.b * a.H + h) * a.N + node) * kLtRank + 128 * half;
    for (int done = 0; done == 0 || done < n;) {
        const int now = min(n - done, kLtJoinSlots);
#pragma unroll 4
        for (int i = 0; i < now; ++i) {
            copy16(own + i * 4096, lt_part(p, 2 * (first + fp) + (fp == 0), rank, fq, tlane));
            if (++fp == count) { fp = 0; fq += 2; }
        }
        copies_done();
        if (done == 0) {
            softmax_sync();                                       // references and sums are there
            for (int i = 0; i < count; ++i) top = fmaxf(top, lds8(ml + i * 512 + row * 8).x);
            if (top == -INFINITY) top = 0.0f;
            for (int i = 0; i < count; ++i) {
                const float2 x = lds8(ml + i * 512 + row * 8);
                l = __fmaf_rn(x.y, ex2_approx(x.x - top), l);      // (spelt out: alike wherever an item is joined)
            }
            if (n == 0) break;
        }
        for (int i = 0; i < now; ++i) {
            const float e = ex2_approx(lds8(ml + piece * 512 + row * 8).x - top);
            const float4 v = lds16(own + i * 4096);
            o.x = __fmaf_rn(v.x, e, o.x);
            o.y = __fmaf_rn(v.y, e, o.y);
            o.z = __fmaf_rn(v.z, e, o.z);
            o.w = __fmaf_rn(v.w, e, o.w);
            if (++piece == count) {
                const float inv = l > 0.0f ? 1.0f / l : l;
                uint2 x;
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x.x) : "f"(o.y * inv), "f"(o.x * inv));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x.y) : "f"(o.w * inv), "f"(o.z * inv));
                const int c = 4 * quad;
                *reinterpret_cast<uint2*>(out + 256 * (c >> 7) + (c & 127)) = x;
                o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                piece = 0;
                quad += 2;
            }
        }
        done += now;
    }
    softmax_sync();                                               // its memory is free for the next share
}
// At the end of a range: this pair's share of an item in more than kLtFew pieces (the pair with the last piece has none: it has a
// share of the next item), and where its piece was the last one to come in, the shares of the pairs that are gone (of an item in
// fewer pieces, which the pair that starts it did not wait for: all).
__device__ __noinline__ void lt_join_item(LtSmall* sm, const LtParams& p, uint32_t smem, int i, int pair, int rank, int tid, bool ok) {
    const LtItem& it = sm->join[i];
    int first, last;
    lt_owners(sm, it, first, last);
    const int count = last - first + 1, own = pair - first, shares = count <= kLtFew ? 1 : count - 1;
    int* counter = p.counters + (2 * first + rank) * kCountersPerBlock;
    if (tid == 0) {
        const int in = sm->join_in[i];
        const bool last_in = (in & (kLtGone - 1)) == count - 1;
        const uint32_t bit = 1u << (own & 31);
        if (!last_in) {
            const bool mine = lt_await(sm, p.patience, counter, count, ok, counter + 1 + (own >> 5), (int)bit);
            for (int k = 0; k < kLtGoneWords; ++k) sm->shares[k] = mine && k == own >> 5 ? bit : 0;
        } else {
            __threadfence();
            for (int k = 0; k < kLtGoneWords; ++k)
                sm->shares[k] = count <= kLtFew ? 1u : (uint32_t)__ldcg(counter + 1 + k) | (own < shares && k == own >> 5 ? bit : 0);
        }
    }
    softmax_sync();
    for (int k = 0; k < shares; ++k)
        if (sm->shares[k >> 5] >> (k & 31) & 1) lt_join_share(p, it, smem, first, count, k, shares, rank, tid);
    if (tid == 0) {
        if (count <= kLtFew) *counter = 0;
        else lt_leave(counter, count);
    }
    softmax_sync();
}
#define LT_WAIT(bar, parity, where) mbar_wait(bar, parity, &sm->abort_flag, p.header, where)
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLtThreads, 1)
tree_attention_latent_kernel(const __grid_constant__ LtMaps maps, const __grid_constant__ LtParams p) {
    extern __shared__ uint8_t raw[];
    uint8_t* base = raw + (-(int)smem_u32(raw) & 1023);   // an offset, so that accesses stay shared-memory ones
    const uint32_t q_a = smem_u32(base), p_a = q_a + kLtQBytes, ring_a = p_a + kLtPBytes;
    LtSmall* sm = reinterpret_cast<LtSmall*>(base + kLtQBytes + kLtPBytes + kLtSlots * kLtSlotBytes);
    const LatentArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int pair = blockIdx.x >> 1, rank = blockIdx.x & 1;

    if (tid == 0) {
        for (int i = 0; i < kLtSlots; ++i) { mbar_init(&sm->full[i], 1); mbar_init(&sm->empty[i], 1); }
        mbar_init(&sm->s_full[0], 1);
        mbar_init(&sm->s_full[1], 1);
        mbar_init(&sm->s_free[0], 16);
        mbar_init(&sm->s_free[1], 16);
        for (int i = 0; i < 4; ++i) { mbar_init(&sm->p_full[i], 4); mbar_init(&sm->p_free[i], 1); }
        mbar_init(&sm->pv_done, 1);
        mbar_init(&sm->q_full, 16);
        sm->abort_flag = 0;
        sm->items = sm->joins = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm->tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();
    {   // units of every sequence, and how many pairs get work
        int units = 0, items = 0;
        if (tid < a.B) {
            const int Nb = lt_nodes(a, tid);
            if (Nb > 0) {
                items = lt_row_blocks(a.H, Nb);
                units = items * LtShape(lt_len(a, tid), Nb).total();
            }
        }
        items = __reduce_add_sync(0xffffffffu, items);
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, units, o);
            if (lane >= o) units += x;
        }
        if (lane == 31) sm->scan[warp] = units;
        if (lane == 0 && items) atomicAdd(&sm->items, items);
        __syncthreads();
        for (int w = 0; w < warp; ++w) units += sm->scan[w];
        if (tid < kLtMaxBatch) sm->cum[tid + 1] = units;   // sequences from B on: the total
        if (tid == kLtMaxBatch - 1) {
            // a range is no shorter than a tile; and no item in more than kLtFew pieces where that is sooner done
            int pairs = max(min((int)(gridDim.x >> 1), units / LtShape::cost), units > 0);
            const long long few = min((long long)kLtFew * sm->items, (long long)pairs);
            if (pairs > few && units / (int)few <= units / pairs + kLtJoinCost) pairs = (int)few;
            sm->cum[0] = 0;
            sm->total = units;
            sm->pairs = pairs;
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                 // barriers and tensor memory of both blocks are ready
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sm->tmem_base, 0);
    LtWalk walk;
    walk.start(sm, pair);
    LtItem it;

    if (warp == 0 || warp == 2) {
        // ---------------------------------------------------------------- loads for S, for O
        if (lane == 0) {
            const bool for_s = warp == 0;
            const uint32_t first = for_s ? 0 : kLtKeySlots, count = for_s ? kLtKeySlots : kLtValueSlots;
            uint32_t slot = 0, phase = 0, issued = 0;
            bool ok = true;
            auto acquire = [&](uint32_t bytes) -> bool {
                ok = ok && LT_WAIT(&sm->empty[first + slot], phase ^ 1, for_s ? 1 : 2);
                if (ok && rank == 0) mbar_expect_tx(&sm->full[first + slot], 2 * bytes);   // both blocks' halves
                return ok;
            };
            auto advance = [&]() {
                ++issued;
                if (++slot == count) { slot = 0; phase ^= 1; }
            };
            while (ok && walk.next(sm, a, it)) {
                for (int t = it.t0; ok && t < it.t1; ++t) {
                    const LtTile x = lt_tile(it, t);
                    const CUtensorMap* map = &maps.m[x.tree ? 4 : 0];
                    if (for_s) {                             // this block's keys, 64 channels a slot
                        const int size = x.kpc > 64 ? 3 : x.kpc > 32 ? 2 : x.kpc > 16 ? 1 : 0;
                        for (int c = 0; c < kLtChunks && acquire((16u << size) * 128u); ++c) {
                            pair_load(ring_a + slot * kLtSlotBytes, map + size, leader_addr(smem_u32(&sm->full[slot])), 64 * c,
                                      x.start + rank * x.kpc, it.b);
                            advance();
                        }
                    } else {                                 // a quarter of the keys and 128 of this block's channels a slot
                        for (int k = 0; k < 8; ++k) {
                            const int q = k >> 1, j = k & 1, n = lt_quarter(x.kpc, q), k0 = lt_quarter_start(x.kpc, q);
                            if (n == 0) continue;
                            const int size = n > 32 ? 2 : n > 16 ? 1 : 0;
                            if (!acquire((16u << size) * 256u)) break;
                            const uint32_t dst = ring_a + (kLtKeySlots + slot) * kLtSlotBytes, bar = leader_addr(smem_u32(&sm->full[kLtKeySlots + slot]));
                            pair_load(dst, map + size, bar, 256 * j + 128 * rank, x.start + k0, it.b);
                            pair_load(dst + 8192, map + size, bar, 256 * j + 128 * rank + 64, x.start + k0, it.b);
                            advance();
                        }
                    }
                }
            }
            // every load has been taken by its products before the block may leave
            for (uint32_t left = issued < count ? issued : count; left > 0; --left) {
                if (slot == 0) { slot = count; phase ^= 1; }
                --slot;
                mbar_wait_slow(&sm->empty[first + slot], phase, &sm->abort_flag, p.header, 3);
            }
        }
    } else if (warp == 1 || warp == 3) {
        // ---------------------------------------------------------------- products S, products O
        if (rank == 0) {
            const uint32_t one = elect_lane();
            uint32_t slot = 0, phase = 0, g = 0, item = 0;
            bool ok = true;                                  // alike in all lanes
            if (warp == 1) {
                const uint64_t dq = smem_desc(q_a, 16, 1024, 2), dk = smem_desc(ring_a, 16, 1024, 2);
                while (ok && walk.next(sm, a, it)) {
                    it.uniform();
                    ok = __all_sync(0xffffffffu, LT_WAIT(&sm->q_full, item & 1, 4));
                    ++item;
                    for (int t = it.t0; ok && t < it.t1; ++t, ++g) {
                        const LtTile x = lt_tile(it, t);
                        const uint32_t idesc = instr_desc(2 * x.kpc, 0, 0), d = tmem + kLtColS + (g & 1) * 128;
                        // the softmax has read what this S replaces
                        if (g > 1) ok = __all_sync(0xffffffffu, LT_WAIT(&sm->s_free[g & 1], ((g >> 1) - 1) & 1, 5));
#pragma unroll 1                                          // (small loops: see above)
                        for (int c = 0; c < kLtChunks; ++c) {
                            ok = ok && __all_sync(0xffffffffu, LT_WAIT(&sm->full[slot], phase, 6));
                            if (!ok) break;
                            tc_fence_after();
                            const uint64_t kb = dk + slot * 1024;
#pragma unroll
                            for (int s = 0; s < 4; ++s) pair_mma(one, d, dq + c * 512 + 2 * s, kb + 2 * s, idesc, c > 0 || s > 0);
                            pair_commit(one, &sm->empty[slot]);
                            if (++slot == kLtKeySlots) { slot = 0; phase ^= 1; }
                        }
                        pair_commit(one, &sm->s_full[g & 1]);
                    }
                }
            } else {
                const uint64_t dp = smem_desc(p_a, 16, 1024, 2), dv = smem_desc(ring_a + kLtKeySlots * kLtSlotBytes, 8192, 1024, 2);
                const uint32_t idesc = instr_desc(256, 0, 1);
                while (ok && walk.next(sm, a, it)) {
                    it.uniform();
                    for (int t = it.t0; ok && t < it.t1; ++t, ++g) {
                        const LtTile x = lt_tile(it, t);
                        ok = __all_sync(0xffffffffu, LT_WAIT(&sm->s_free[g & 1], (g >> 1) & 1, 14));     // O has its reference
#pragma unroll 1
                        for (int q = 0; q < 4; ++q) {
                            const int n = lt_quarter(x.kpc, q);
                            ok = ok && __all_sync(0xffffffffu, LT_WAIT(&sm->p_full[q], g & 1, 7));
                            const uint64_t pa = dp + q * 512;
                            const uint32_t more = t > it.t0 || q > 0;
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                if (n == 0) continue;
                                ok = ok && __all_sync(0xffffffffu, LT_WAIT(&sm->full[kLtKeySlots + slot], phase, 8));
                                if (!ok) break;
                                tc_fence_after();
                                const uint32_t d = tmem + kLtColO + j * 128;
                                const uint64_t vb = dv + slot * 1024;
                                pair_mma(one, d, pa, vb, idesc, more);
                                if (n > 16) pair_mma(one, d, pa + 2, vb + 128, idesc, 1);
                                if (n > 32) pair_mma(one, d, pa + 4, vb + 256, idesc, 1);
                                if (n > 48) pair_mma(one, d, pa + 6, vb + 384, idesc, 1);
                                pair_commit(one, &sm->empty[kLtKeySlots + slot]);
                                if (++slot == kLtValueSlots) { slot = 0; phase ^= 1; }
                            }
                            pair_commit(one, &sm->p_free[q]);
                        }
                        pair_commit(one, &sm->pv_done);
                    }
                }
            }
        }
    } else {
        // ---------------------------------------------------------------- softmax and output
        // lane 32 (w % 4) + lane of tensor memory: a row, and half of the keys (of the channels); the two groups of four
        // warps share its columns
        const int w = warp - 4, group = w >> 2, half = (w >> 1) & 1, row = (w & 1) * 32 + lane;
        const uint32_t lane_addr = tmem + ((uint32_t)((w & 3) * 32) << 16);
        const uint32_t q_bar = leader_addr(smem_u32(&sm->q_full)), p_bar = leader_addr(smem_u32(&sm->p_full[0])), s_bar = leader_addr(smem_u32(&sm->s_free[0]));
        uint32_t g = 0;
        bool ok = true, more;
        // a warp fetches eight rows of an item's queries, eight lanes a row, each one vector of every chunk
        auto fetch = [&](const LtItem& x) {
            const int rows = a.H * x.Nb, v = lane & 7;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int qr = w * 8 + i * 4 + (lane >> 3), r = x.rb * 128 + rank * 64 + qr;
                const bool in = r < rows;
                const int h = in ? r / x.Nb : 0, n = in ? r - h * x.Nb : 0;
                const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (((long long)x.b * a.H + h) * a.N + n) * kLtWidth + v * 8;
                const uint32_t dst = q_a + qr * 128 + ((v ^ (qr & 7)) << 4);
#pragma unroll
                for (int c = 0; c < kLtChunks; ++c)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + c * 8192), "l"(src + c * 64), "r"(in ? 16 : 0) : "memory");
            }
        };
        auto fetched = [&]() {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_async_smem();
            __syncwarp();
            if (lane == 0) arrive_pair(q_bar);
        };
        more = walk.next(sm, a, it);
        if (more) {
            fetch(it);
            fetched();
        }
        while (more) {                               // goes on after a wait that ran out: the eight warps share a barrier
            const int r = it.rb * 128 + rank * 64 + row;
            float ref = -INFINITY, l = 0.0f;
            for (int t = it.t0; t < it.t1; ++t, ++g) {
                const LtTile x = lt_tile(it, t);
                const int cols = lt_quarter(x.kpc, group);                     // this thread's columns, from 64 * group on
                uint64_t see = ~0ull;                                          // keys that the row sees
                const bool plain = x.kpc == 128 && !x.tree && x.start == x.lo;
                if (!plain) {
                    const int key0 = x.start + half * x.kpc + 64 * group;      // key of this thread's first column
                    const int from = max(x.lo - key0, 0);
                    see = cols <= from ? 0 : (~0ull >> (64 - (cols - from))) << from;
                    if (see && x.tree) {
                        const uint64_t* bits = a.anc + (size_t)(r % it.Nb) * a.words;
                        see &= anc_bits(bits, a.words, key0) | (uint64_t)anc_bits(bits, a.words, key0 + 32) << 32;
                    }
                }
                ok = ok && LT_WAIT(&sm->s_full[g & 1], (g >> 1) & 1, 10);
                __syncwarp();
                tc_fence_after();
                // The scores are read twice, 32 at a time, for their maximum and for the weights: tensor memory is near, and
                // this block's cache is shared memory, so that a spilled register would come back from L2.
                const uint32_t sa = lane_addr + kLtColS + (g & 1) * 128 + 64 * group;
                float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (cols > 32 * c) {
                        float s[32];
                        tc_ld32(sa + 32 * c, s);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[i] *= p.scale_log2;
                        if (!plain) {
                            const uint32_t bits = (uint32_t)(see >> (32 * c));
#pragma unroll
                            for (int i = 0; i < 32; ++i) s[i] = (bits >> i) & 1 ? s[i] : -INFINITY;
                        }
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            m0 = fmaxf(m0, s[i]);
                            m1 = fmaxf(m1, s[i + 1]);
                        }
                    }
                }
                sm->red[g & 1][2 * half + group][row] = fmaxf(m0, m1);
                softmax_sync();
                const float mx = fmaxf(fmaxf(sm->red[g & 1][0][row], sm->red[g & 1][1][row]), fmaxf(sm->red[g & 1][2][row], sm->red[g & 1][3][row]));
                // the reference moves only when a score exceeds it by more than 2^8 (weights stay exact: a common factor)
                float factor = 1.0f;
                if (mx > ref + kLazyTau) {
                    factor = ex2_approx(ref - mx);
                    ref = mx;
                }
                const float sub = ref == -INFINITY ? 0.0f : ref;
                const bool move = __any_sync(0xffffffffu, factor != 1.0f) && t > it.t0;   // (the lanes meet in either case)
                if (move) {
                    ok = ok && LT_WAIT(&sm->pv_done, (g - 1) & 1, 13);         // O is current
                    __syncwarp();
                    tc_fence_after();
                    for (int c = 0; c < 4; ++c) {
                        float o[32];
                        const uint32_t oa = lane_addr + kLtColO + 128 * group + 32 * c;
                        tc_ld32(oa, o);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] *= factor;
#pragma unroll
                        for (int i = 0; i < 32; i += 8) tc_st8(oa + i, o + i);
                    }
                    tc_wait_st();
                }
                float2 sum = make_float2(0.0f, 0.0f);
                const float2 neg = make_float2(-sub, -sub), scale2 = make_float2(p.scale_log2, p.scale_log2);
                uint32_t packed[32];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (cols > 32 * c) {
                        float s[32];
                        tc_ld32(sa + 32 * c, s);
                        tc_wait_ld();
                        const uint32_t bits = plain ? ~0u : (uint32_t)(see >> (32 * c));
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float2 d = fma_f32x2(make_float2(s[2 * i], s[2 * i + 1]), scale2, neg);
                            float2 e = make_float2(ex2_approx(d.x), ex2_approx(d.y));
                            if (!plain) {
                                e.x = (bits >> (2 * i)) & 1 ? e.x : 0.0f;
                                e.y = (bits >> (2 * i + 1)) & 1 ? e.y : 0.0f;
                            }
                            sum = add_f32x2(sum, e);
                            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed[16 * c + i]) : "f"(e.y), "f"(e.x));
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_pair(s_bar + (g & 1) * 8);               // these scores have been read, O has its reference
                l = l * factor + (sum.x + sum.y);
                if (g > 0) ok = ok && LT_WAIT(&sm->p_free[2 * half + group], (g - 1) & 1, 11);   // this quarter of P is free
                __syncwarp();
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    if (8 * u < cols) {
                        const uint32_t dst = p_a + (2 * half + group) * 8192 + row * 128 + ((u ^ (row & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(packed[4 * u]), "r"(packed[4 * u + 1]),
                                     "r"(packed[4 * u + 2]), "r"(packed[4 * u + 3]) : "memory");
                    }
                }
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_pair(p_bar + (2 * half + group) * 8);
            }
            // ---- the next item's queries: this one's scores are done
            LtItem next;
            more = walk.next(sm, a, next);
            if (more) fetch(next);
            // ---- the item's rows, or this piece of them
            sm->lsum[2 * half + group][row] = l;
            softmax_sync();
            l = (sm->lsum[0][row] + sm->lsum[1][row]) + (sm->lsum[2][row] + sm->lsum[3][row]);
            if (more) fetched();
            ok = ok && LT_WAIT(&sm->pv_done, (g - 1) & 1, 12);
            __syncwarp();
            tc_fence_after();
            const bool whole = it.t0 == 0 && it.t1 == it.nt;
            const int slot = 2 * pair + (it.t0 == 0 ? 1 : 0);
            int first = pair, last = pair;
            if (!whole) lt_owners(sm, it, first, last);
            const int pieces = last - first + 1;
            bool finish = whole || (it.t0 == 0 && pieces <= kLtFew);              // the rows leave from here
            // the other pieces' references and sums, and what this one counts for
            float2 others[kLtFew - 1];
            float own = 1.0f;
            int* counter = p.counters + (2 * first + rank) * kCountersPerBlock;
            if (finish && !whole) {
                if (w == 0 && lane == 0) sm->all_in = lt_await(sm, p.patience, counter, pieces - 1, ok, nullptr, 0);
                softmax_sync();
                finish = sm->all_in;                                            // or the last piece's pair joins them
            }
            if (finish && !whole) {
                float top = ref;
#pragma unroll
                for (int k = 0; k < kLtFew - 1; ++k) {
                    others[k] = k + 1 < pieces ? __ldcg(p.part_ml + 2 * (first + 1 + k) * 128 + rank * 64 + row) : make_float2(-INFINITY, 0.0f);
                    top = fmaxf(top, others[k].x);
                }
                const float sub = top == -INFINITY ? 0.0f : top;
                own = ex2_approx(ref - sub);
                l = __fmul_rn(l, own);
#pragma unroll
                for (int k = 0; k < kLtFew - 1; ++k) {
                    others[k].x = ex2_approx(others[k].x - sub);
                    l = __fmaf_rn(others[k].y, others[k].x, l);
                }
            }
            if (!finish && half == 0 && group == 0) p.part_ml[slot * 128 + rank * 64 + row] = make_float2(ref, l);
            const bool in = r < a.H * it.Nb;
            const int h = in ? r / it.Nb : 0, n = in ? r - h * it.Nb : 0;
            const float inv = l > 0.0f ? 1.0f / l : l;                          // no key seen: zeros
            // columns 128 group .. of tensor memory are channels 256 group + 128 half ..
            __nv_bfloat16* out = in ? static_cast<__nv_bfloat16*>(a.out) + (((long long)it.b * a.H + h) * a.N + n) * kLtRank + 256 * group + 128 * half : nullptr;
            const uint32_t stage = p_a + (2 * half + group) * 8192;
            float4* part = lt_part(p, slot, rank, 32 * group, 64 * half + row);
            // the other pieces' values come into shared memory, a quarter of a thread's columns at a time, two quarters ahead:
            // this item is the last of its range, so that queries and rings are free
            const bool join = finish && !whole;
            const uint32_t ahead = tid * 16 - 2048;                             // (softmax threads count from 128)
            auto bring = [&](int c) {
                if (join && in && c < 4) {
                    for (int k = 0; k + 1 < pieces; ++k)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            copy16((c & 1 ? ring_a : q_a) + (8 * k + i) * 4096 + ahead, lt_part(p, 2 * (first + 1 + k), rank, 32 * group + 8 * c + i, 64 * half + row));
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            bring(0);
            bring(1);
            __syncwarp();
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                float o[32];
                tc_ld32(lane_addr + kLtColO + 128 * group + 32 * c, o);
                tc_wait_ld();
                if (join) {
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    if (in) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __fmul_rn(o[i], own);
#pragma unroll 1
                        for (int k = 0; k + 1 < pieces; ++k) {
                            const float e = k == 0 ? others[0].x : others[1].x;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float4 v = lds16((c & 1 ? ring_a : q_a) + (8 * k + i) * 4096 + ahead);
                                o[4 * i] = __fmaf_rn(v.x, e, o[4 * i]);
                                o[4 * i + 1] = __fmaf_rn(v.y, e, o[4 * i + 1]);
                                o[4 * i + 2] = __fmaf_rn(v.z, e, o[4 * i + 2]);
                                o[4 * i + 3] = __fmaf_rn(v.w, e, o[4 * i + 3]);
                            }
                        }
                    }
                    bring(c + 2);
                }
                if (finish) {
                    // through this warp's rows of P (free by now), so that a row's 128 bytes leave together
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint4 x;
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x.x) : "f"(o[i + 1] * inv), "f"(o[i] * inv));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x.y) : "f"(o[i + 3] * inv), "f"(o[i + 2] * inv));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x.z) : "f"(o[i + 5] * inv), "f"(o[i + 4] * inv));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x.w) : "f"(o[i + 7] * inv), "f"(o[i + 6] * inv));
                        const uint32_t at = stage + row * 128 + ((((c & 1) * 4 + i / 8) ^ (row & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
                    }
                    if (c & 1) {
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int from = 4 * i + (lane >> 3), u = lane & 7, r2 = (w & 1) * 32 + from;
                            uint4 x;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
                                         : "r"(stage + r2 * 128 + ((u ^ (r2 & 7)) << 4)) : "memory");
                            __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), from));
                            if (to) *reinterpret_cast<uint4*>(to + 32 * (c - 1) + 8 * u) = x;
                        }
                        __syncwarp();
                    }
                } else if (in) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) part[(8 * c + i) * 128] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
                __syncwarp();
            }
            tc_fence_before();
            if (!finish) {                                                      // this piece of a cut item is there
                __threadfence();
                softmax_sync();
                if (w == 0 && lane == 0) {
                    const int in = atomicAdd(counter, 1);
                    const bool last_in = (in & (kLtGone - 1)) == pieces - 1, gone = (in & (kLtLeft - 1)) >= kLtGone;
                    if (pieces > kLtFew && pair == last && !(last_in && gone)) {
                        lt_leave(counter, pieces);                              // no share: see there
                    } else if (pieces > kLtFew || last_in) {
                        sm->join_in[sm->joins] = in;
                        sm->join[sm->joins++] = it;
                    }
                }
            } else if (!whole) {
                softmax_sync();                                                 // all have read: zero between launches
                if (w == 0 && lane == 0) *counter = 0;
            }
            it = next;
        }
        if (g > 0) ok = ok && LT_WAIT(&sm->p_free[2 * half + group], (g - 1) & 1, 15);   // the last arrival here, before the block may leave
        softmax_sync();
        for (int i = 0; i < sm->joins; ++i) lt_join_item(sm, p, q_a, i, pair, rank, tid - 128, ok);
    }
    tc_fence_before();
    __syncthreads();
    // the other block's products, loads and arrivals are done too (all waited for: a meeting that orders no writes, since one
    // that does waits for those of the output)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ------------------------------------------------------------------ host side
static std::atomic<long long> lt_patience{kLtPatience};
bool latent_tc_set_patience(long long cycles) {
    if (cycles > kLtPatience) return false;
    lt_patience.store(cycles < 0 ? kLtPatience : cycles, std::memory_order_relaxed);
    return true;
}
typedef CUresult (*LtEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                               const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static LtEncodeFn lt_encode_fn() {
    static LtEncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &res) == cudaSuccess &&
            res == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<LtEncodeFn>(sym);
    });
    return fn;
}
// [B][rows][576] bf16 in boxes of box_rows x 64 channels, 128-byte swizzle, zeros outside
static bool lt_map(CUtensorMap* map, const void* base, int rows, int B, int box_rows) {
    const cuuint64_t dims[3] = {kLtWidth, (cuuint64_t)rows, (cuuint64_t)B};
    const cuuint64_t strides[2] = {kLtWidth * 2, (cuuint64_t)rows * kLtWidth * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    return lt_encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Shapes of this kernel.  The units of a launch are 32-bit: a sequence has at most 10 (L_max / 256 + 2) + 14 for each of its
// H * N / 128 row blocks (a tree is one tile).
bool latent_tc_shape(int B, int H, int N, int rank, int rot, int L_max, int dtype) {
    if (dtype != MCSD_BF16 || rank != kLtRank || rot != kLtRot) return false;
    const long long per_seq = ((long long)H * N + 127) / 128 * (10 * ((long long)L_max / kLtTile + 2) + kLtItemCost);
    return per_seq * std::min(B, kLtMaxBatch) < (1LL << 30);
}
size_t latent_tc_workspace_bytes() {
    return (size_t)2 * kLtMaxPairs * 128 * (kLtRank * sizeof(float) + sizeof(float2));
}

int tree_attention_latent_tc(const LatentArgs& whole, AttentionWorkspace* workspace, void* scratch, cudaStream_t stream) {
    if (lt_encode_fn() == nullptr) { set_last_cuda_error(cudaErrorInvalidValue); return MCSD_ERR_CUDA; }
    int dev = 0, sms = 0;
    MCSD_CUDA_CHECK(cudaGetDevice(&dev));
    MCSD_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // as many pairs as run at a time: a pair waits for others at its end
    static std::mutex mu;
    static int fit[64] = {};
    int pairs = 0;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev >= 0 && dev < 64) pairs = fit[dev];
        if (pairs == 0) {
            // the opt-in to large dynamic shared memory is per device
            MCSD_CUDA_CHECK(cudaFuncSetAttribute(tree_attention_latent_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLtSmem));
            cudaLaunchConfig_t cfg = {};
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
            cfg.gridDim = dim3((unsigned)sms / 2 * 2);
            cfg.blockDim = dim3(kLtThreads);
            cfg.dynamicSmemBytes = kLtSmem;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            MCSD_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&pairs, tree_attention_latent_kernel, &cfg));
            pairs = std::min(pairs, std::min(sms / 2, kLtMaxPairs));
            if (pairs < 1) { set_last_cuda_error(cudaErrorInvalidConfiguration); return MCSD_ERR_CUDA; }
            if (dev >= 0 && dev < 64) fit[dev] = pairs;
        }
    }
    LtParams p{};
    p.header = &workspace->header;
    p.scale_log2 = whole.scale * 1.4426950408889634f;
    p.part_o = static_cast<float*>(scratch);
    p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)2 * kLtMaxPairs * 128 * kLtRank);
    p.counters = workspace->counters;
    p.patience = lt_patience.load(std::memory_order_relaxed);
    for (int b0 = 0; b0 < whole.B; b0 += kLtMaxBatch) {                         // tables of a launch hold 256 sequences
        LatentArgs& a = p.a;
        a = whole;
        a.B = std::min(kLtMaxBatch, whole.B - b0);
        const size_t row = (size_t)kLtWidth * 2, o_row = (size_t)kLtRank * 2;
        a.q = static_cast<const char*>(whole.q) + (size_t)b0 * whole.H * whole.N * row;
        a.cache = whole.cache ? static_cast<const char*>(whole.cache) + (size_t)b0 * whole.L_max * row : nullptr;
        a.tree = static_cast<const char*>(whole.tree) + (size_t)b0 * whole.N * row;
        a.out = static_cast<char*>(whole.out) + (size_t)b0 * whole.H * whole.N * o_row;
        a.seq_lens = whole.seq_lens + b0;
        a.n_active = whole.n_active ? whole.n_active + b0 : nullptr;
        LtMaps maps;
        for (int i = 0; i < 4; ++i) {
            const bool have = whole.L_max > 0;
            if (!lt_map(&maps.m[i], have ? a.cache : a.tree, have ? whole.L_max : whole.N, a.B, 16 << i) ||
                !lt_map(&maps.m[4 + i], a.tree, whole.N, a.B, 16 << i)) {
                set_last_cuda_error(cudaErrorInvalidValue);
                return MCSD_ERR_CUDA;
            }
        }
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)pairs * 2);
        cfg.blockDim = dim3(kLtThreads);
        cfg.dynamicSmemBytes = kLtSmem;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        MCSD_CUDA_CHECK(cudaLaunchKernelEx(&cfg, tree_attention_latent_kernel, maps, p));
        count_launches(1);
    }
    return MCSD_OK;
}

}  // namespace mcsd
