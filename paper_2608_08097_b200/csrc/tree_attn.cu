// Attention of a tree of drafted tokens over the working set, on the 5th-generation tensor cores.
//
// A query row is (node t, query head a).  It sees the history in the row's columns (positions below seq_len) and, in the
// tree buffer, its ancestors and itself.  The structure is that of the chain attention (attn_tc.cu, whose pieces in
// tc_common.cuh it shares): work item = (request, KV head, row group, split of the column list), one thread block, the
// group's query rows as the M rows of every MMA, tiles of four 16-key blocks in a ring of six 32 KiB stages, the queries
// in shared memory too (by TMA, read by every Q K^T from there), warp 0 the TMA producer, warps 1 and 2 the issuers of Q K^T and P V, the others softmax with one thread per MMA row.  What differs:
//   - The keys are a list of blocks: the row's visible history blocks, then the blocks of the tree buffer, which comes
//     through a tensor map of its own ([token][head][K, V] -> the same 8 KiB block image, nodes past n_tree read as
//     zero).  The producer compacts: columns that are empty or lie past seq_len take no place in a tile and move no
//     bytes, so a mostly empty resident table costs nothing; the other warps count the same columns meanwhile, because
//     every role needs the number of tiles.
//   - A block's visible keys are a 16-bit mask per row: a prefix for history blocks (the same for all rows), the node's
//     ancestor bits for tree blocks.  Ancestors come from the parents by pointer doubling (six rounds for 64 nodes).
//   - Key rows that no query may see hold anything, NaN included, and 0 x NaN is NaN in P V: before P is handed to the
//     tensor core, the softmax warps overwrite those V rows with zeros in shared memory (masked tiles only).
//   - Up to 256 query rows share a thread block (two MMAs of 128 rows per tile); more are cut into row groups of equal
//     size, neighbouring thread blocks that read the same entries at the same time, so that all but one come from L2.
//   - Splits of a row merge inside a thread-block cluster where a cluster reaches far enough, else in a second launch.
// Algorithmic traffic: 8 KiB per (request, KV head, visible column), 512 B per (node, KV head), plus Q, O and lse.
// Precision: logits, the running maximum and sum and the accumulators are fp32.  The softmax weights go to P V as bf16 (half a
// step, 2^-8 of a weight), because both operands of one tcgen05.mma kind::f16 have the same type and V is bf16; the sum that
// divides them is of the unrounded ones.  Against 64 bits outputs are off by 0.2 % of their norm, 0.17 % with fp32 weights.
// What bounds it (32 query and 8 KV heads, per call in a replayed graph): HBM for long lists, 86.4 us at 6.2 TB/s for 2
// requests x 4,098 columns; HBM and some 7 us of launch, first loads, epilogue and merge for 16 requests x 130 columns
// under 16 nodes, 28.1 us (4.9 TB/s); under 64 nodes, 42.7 us, the softmax and the products between which a tile goes back and
// forth: of its 2,050 cycles the exponential unit is busy for 1,024 (two softmax warps per scheduler, 64 ex2 each at 8 cycles) and
// the tensor core for 1,280.  That is sixteen products of 128 x 64 x 16 with both operands in shared memory, 48 cycles each (32
// of arithmetic; reading the operands' 6 KiB takes 48), and eight of 128 x 128 x 16 at 64.  Tiles of 128 keys, whose logits fit
// into the tensor memory only once beside the accumulators, take 47.4 us.
#include <cuda.h>
#include <math_constants.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace oasis {

// Warp sets of four softmax warps: one, or two that take alternate tiles (65 to 128 rows) or half the rows each (PAIR).
__host__ __device__ constexpr int tr_sets(int mma_m, int copies, bool pair) { return pair ? 2 : at_softmax_sets(mma_m, copies); }
__host__ __device__ constexpr int tr_threads(int mma_m, int copies, bool pair)    // producer, two MMA issuers, softmax warps
{
    return 96 + 128 * tr_sets(mma_m, copies, pair);
}
// The query rows in shared memory: [dim half][MMA rows][128 B], 128-byte swizzle.
__host__ __device__ constexpr int tr_rows(int mma_m, bool pair) { return pair ? 256 : mma_m; }
__host__ __device__ constexpr int tr_stages(bool pair) { return pair ? 5 : 6; }      // of 32 KiB; with the queries 224 KiB at most
constexpr int kTrMaxCluster = 8;
constexpr int32_t kTreeTag = 0x40000000;                    // tile_blk: kTreeTag + i = block i of the tree buffer
// Behind the ring: 512 B of barriers and tile ids, two table windows, the producer's block queue, ancestor masks.
constexpr int kTrQueue = 64;
constexpr int kTrUp = 8 * (2 * kAtMaxStages + 2 * kAtSBufs + 4) + 16 * kAtMaxStages;   // parents: behind barriers and tile ids
constexpr int kTrPlain = kTrUp + OASIS_MAX_TREE;                                       // one word per stage
constexpr int kTrMisc = 512 + 2 * kWinBytes + kTrQueue * 8 + OASIS_MAX_TREE * 8;
__host__ __device__ constexpr int tr_smem(int mma_m, bool pair)
{
    return 1024 + tr_rows(mma_m, pair) * kRowBytes + tr_stages(pair) * kAtStageBytes + kTrMisc;
}
static_assert(kTrPlain + 4 * kAtMaxStages <= 512 && tr_smem(128, false) <= 232448 && tr_smem(128, true) <= 232448, "shared memory of a thread block");

struct TreeAttnParams {
    const int32_t *slot_tbl, *blk_tbl, *seq_len, *parent, *n_nodes;
    uint8_t *out;
    float *lse;
    float *part_o;      // [items][rows per group][128] fp32 (split runs only)
    float *part_lse;    // [items][rows per group]      log2 domain
    int32_t *err;
    float scale_log2;
    int T, Hq, Hkv, G, n_cols, R, n_splits, cols_per_split, n_groups, group_rows;      // group_rows: a multiple of G
    long long n_slots;  // bounds-check build: slots of the working-set pool (else unused)
};

// Values from the same shared-memory place of thread block `rank` of the cluster.
__device__ __forceinline__ uint32_t at_rank(const void *place, uint32_t rank)
{
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(place)), "r"(rank));
    return addr;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier()       // every thread of every block of the cluster
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ bool block_seen(int blk, int len) { return blk >= 0 && (long long)blk * kBlock < len; }

// PAIR: 129 to 256 query rows, two MMAs of 128 rows per tile.  Each set of softmax warps owns 128 rows and takes every tile;
// both have two S buffers and an O accumulator, which fills the tensor memory.
template <int MMA_M, int COPIES, bool PAIR, bool CLUSTER>
__global__ void __launch_bounds__(tr_threads(MMA_M, COPIES, PAIR), 1)
tree_attn_tc_kernel(const __grid_constant__ CUtensorMap pool_map, const __grid_constant__ CUtensorMap tree_map,
                    const __grid_constant__ CUtensorMap q_map, const TreeAttnParams p)
{
    constexpr int RPC = MMA_M / COPIES;                     // MMA rows per copy of the query rows
    constexpr int LANES = MMA_M / 4;                        // lanes of each softmax warp that hold an MMA row
    constexpr int BPC = kAtTileCols / COPIES;               // blocks of a tile each copy handles
    static_assert(!PAIR || (MMA_M == 128 && COPIES == 1), "two tiles of 128 query rows");
    constexpr int SETS = PAIR ? 1 : at_softmax_sets(MMA_M, COPIES);    // softmax warp sets that take alternate tiles
    constexpr int HALVES = PAIR ? 2 : 1;                    // MMA tiles of query rows
    constexpr int SBUFS = PAIR ? 2 : kAtSBufs;              // S / P buffers in tensor memory (of each half)
    constexpr int QHALF = tr_rows(MMA_M, PAIR) * 128;       // bytes of the query rows' first 64 dims
    constexpr int THREADS = tr_threads(MMA_M, COPIES, PAIR);
    constexpr int STAGES = tr_stages(PAIR);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base - smem_u32(smem_raw));
    uint8_t *const kv_ptr = base_ptr + 2 * QHALF;                    // [stages][32 KiB]
    const uint32_t kv_u32 = base + 2 * QHALF;
    uint8_t *misc = kv_ptr + (size_t)STAGES * kAtStageBytes;
    const uint32_t bar_u32 = smem_u32(misc);
    auto bar_full = [&](int s) { return bar_u32 + 8u * s; };
    auto bar_empty = [&](int s) { return bar_u32 + 8u * (kAtMaxStages + s); };
    auto bar_s_full = [&](int a) { return bar_u32 + 8u * (2 * kAtMaxStages + a); };
    auto bar_p_full = [&](int a) { return bar_u32 + 8u * (2 * kAtMaxStages + kAtSBufs + a); };
    const uint32_t bar_q = bar_u32 + 8u * (2 * kAtMaxStages + 2 * kAtSBufs);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(misc + 8 * (2 * kAtMaxStages + 2 * kAtSBufs + 2));
    int32_t *s_count = reinterpret_cast<int32_t *>(misc + 8 * (2 * kAtMaxStages + 2 * kAtSBufs + 2) + 4);
    int32_t *tile_blk = reinterpret_cast<int32_t *>(misc + 8 * (2 * kAtMaxStages + 2 * kAtSBufs + 4));   // [stages][4]
    int32_t *win = reinterpret_cast<int32_t *>(misc + 512);                                             // two table windows
    int2 *queue = reinterpret_cast<int2 *>(misc + 512 + 2 * kWinBytes);                                  // (block, slot)
    unsigned long long *anc = reinterpret_cast<unsigned long long *>(queue + kTrQueue);                   // [T] ancestor masks
    int32_t *plain = reinterpret_cast<int32_t *>(misc + kTrPlain);                                        // [stages]: all keys visible
    int8_t *up = reinterpret_cast<int8_t *>(misc + kTrUp);                                                // [T]

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // (row groups of the same entries side by side; a row's splits, where they are a cluster)
    const int grp = CLUSTER ? (blockIdx.x / p.n_splits) % p.n_groups : blockIdx.x % p.n_groups;
    const int split = CLUSTER ? blockIdx.x % p.n_splits : (blockIdx.x / p.n_groups) % p.n_splits;
    const int bh = blockIdx.x / (p.n_groups * p.n_splits);
    const int b = bh / p.Hkv, h = bh % p.Hkv;
    const int row0 = grp * p.group_rows;                             // first query row (node * G + head) of the group
    const int c0 = split * p.cols_per_split;
    const int c1 = min(c0 + p.cols_per_split, p.n_cols);
    const int32_t *slot_row = p.slot_tbl + (long long)bh * p.n_cols;
    const int32_t *blk_row = p.blk_tbl + (long long)bh * p.n_cols;
    if (tid == 0) {
        for (int s = 0; s < kAtMaxStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        for (int a = 0; a < kAtSBufs; ++a) { mbar_init(bar_s_full(a), 1); mbar_init(bar_p_full(a), 4); }
        mbar_init(bar_q, 1);
        *s_count = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // This launch may have been brought onto the SMs before the previous one ended: what that wrote is read from here on.  Only then
    // may a launch behind this one (the merge of the splits, the next attention) be brought in the same way: it may read, without
    // a wait of its own, what launches before this one wrote (the scoring of oasis_attn_and_score does).
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 0 && c0 < c1) window_request(smem_u32(win), lane, blk_row, slot_row, c0 + lane, c1);     // (needs no length)
    // every first load is on its way before the first is used: lengths, this thread's column, the parents (warp 2)
    const int n_nodes_raw = p.n_nodes[b], L = p.seq_len[b];
    const int my_col = c0 + tid - 32;
    const int my_blk = warp > 0 && my_col < c1 ? blk_row[my_col] : -1;
    int par[2] = {-1, -1};
    if (warp == 2) {
        if (lane < p.T) par[0] = p.parent[(long long)b * p.T + lane];
        if (lane + 32 < p.T) par[1] = p.parent[(long long)b * p.T + lane + 32];
    }
    const int n_nodes = max(0, min(n_nodes_raw, p.T));
    const int rows = min(min(p.group_rows, p.R - row0), n_nodes * p.G - row0);
    if (rows <= 0) {                                                 // only padding nodes: nothing is read or written
        window_wait();
        return;
    }
    // blocks of the tree buffer that the group's rows may see (ancestors have lower indices), taken by the last split
    const int n_tree_blk = split == p.n_splits - 1 ? (row0 + rows - 1) / p.G / kBlock + 1 : 0;

    // ---- set-up: tensor memory, ancestor masks, number of tiles --------------------------------------------
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();                             // the barriers exist; the producer starts copying right away
    uint32_t tmem_base = 0, tmem_o = 0;
    int n_tiles = 0;
    if (warp != 0) {
        // Meanwhile: warp 1 allocates the tensor memory, warp 2 works out the ancestors, all count the visible columns.
        if (warp == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)kAtTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        int seen = block_seen(my_blk, L);
        for (int c = my_col + THREADS - 32; c < c1; c += THREADS - 32) seen += block_seen(blk_row[c], L);
        seen = __reduce_add_sync(0xffffffffu, seen);
        if (lane == 0 && seen) atomicAdd(s_count, seen);
        if (warp == 2) {
            unsigned long long m[2];
            int u[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = lane + 32 * e;
                u[e] = t < n_nodes && par[e] >= 0 && par[e] < t ? par[e] : -1;
                m[e] = 1ull << t;
            }
#pragma unroll 1
            for (int round = 0; round < 6; ++round) {
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 2; ++e) { anc[lane + 32 * e] = m[e]; up[lane + 32 * e] = (int8_t)u[e]; }
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (u[e] >= 0) { m[e] |= anc[u[e]]; u[e] = up[u[e]]; }
            }
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 2; ++e) anc[lane + 32 * e] = m[e];
        }
        tc_fence_before();
        asm volatile("bar.sync 2, %0;" ::"n"(THREADS - 32) : "memory");
        tc_fence_after();
        n_tiles = (*s_count + n_tree_blk + kAtTileCols - 1) / kAtTileCols;
        tmem_base = *tmem_slot;
        tmem_o = tmem_base + HALVES * SBUFS * kAtTileKeys;
    }

    // After the last tile the K/V ring is idle.  Every accumulator row goes there with its maximum and sum (part = copy or set
    // of the query row), then the warps write whole rows: merged, normalised, coalesced.
    constexpr int PARTS = COPIES * SETS, PITCH = kHeadDim + 4, WRITERS = (THREADS - 96) / 32;
    float *const o_sm = reinterpret_cast<float *>(kv_ptr);           // [PARTS * RPC or 256][PITCH], then maxima and sums
    float *const m_sm = o_sm + 256 * PITCH, *const l_sm = m_sm + 256;
    float *const row_lse = l_sm + 256;                               // clusters: of the block's parts together

    if (warp == 0) {
        // ---------------------------------------------------------------- producer
        // Table entries come 32 columns at a time through two window buffers, one window ahead; the visible ones go into
        // a queue, and every four of them are a tile.
        const uint32_t win_u32 = smem_u32(win);
        bool alive = true;
        int s = 0, head = 0, tail = 0;
        uint32_t ph = 1;                                             // parity of the "empty" phase to wait for
        auto emit = [&](int count) {                                 // the queue's next `count` <= 4 blocks as a tile
            int blk = -1, slot = -1;
            if (lane < count) {
                const int2 e = queue[(head + lane) & (kTrQueue - 1)];
                blk = e.x;
                slot = e.y;
                if (kBoundsCheck && blk < kTreeTag && !in_range(slot, p.n_slots, Bounds{0, 0, p.err}, kErrSlot)) blk = -1;
            }
            head += count;
            if (lane == 0) alive = mbar_wait(bar_empty(s), ph, p.err, 41);
            alive = __shfl_sync(0xffffffffu, (int)alive, 0) != 0;
            if (!alive) return;
            uint8_t *stage = kv_ptr + (size_t)s * kAtStageBytes;
            const uint32_t stage_u32 = kv_u32 + s * kAtStageBytes;
            const unsigned valid = __ballot_sync(0xffffffffu, lane < kAtTileCols && blk >= 0);
            const unsigned full = __ballot_sync(0xffffffffu, lane < kAtTileCols && blk >= 0 && blk < kTreeTag && L - blk * kBlock >= kBlock);
            if (lane < kAtTileCols) tile_blk[s * kAtTileCols + lane] = blk;
            if (lane == 0) plain[s] = full == 0xfu;
            if ((valid & 0xfu) != 0xfu) {
                // a missing block contributes P = 0, which must not meet stale NaN patterns: the warp zeroes its V image
#pragma unroll
                for (int c = 0; c < kAtTileCols; ++c) {
                    if ((valid >> c) & 1u) continue;
                    uint8_t *dst = stage + c * kEntryBytes + (lane >> 4) * kImgGroup + ((lane >> 3) & 1) * kImgHalf + kImgPart + (lane & 7) * 128;
#pragma unroll
                    for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4 *>(dst + j * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_expect_tx(bar_full(s), (uint32_t)__popc(valid) * kEntryBytes);
            __syncwarp();
            if (lane < kAtTileCols && blk >= 0) {
                const uint32_t dst = stage_u32 + lane * kEntryBytes;
                if (blk < kTreeTag) {
                    tma_load_5d(dst, &pool_map, 0, 0, 2 * slot, 0, 0, bar_full(s));
                } else {                                             // the two 8-node groups of a tree block
                    const int t = (blk - kTreeTag) * kBlock;
                    tma_load_5d(dst, &tree_map, 0, t, 2 * h, 0, b, bar_full(s));
                    tma_load_5d(dst + kImgGroup, &tree_map, 0, t + 8, 2 * h, 0, b, bar_full(s));
                }
            }
            ph ^= (s + 1 == STAGES);
            s = (s + 1 == STAGES) ? 0 : s + 1;
        };
        if (lane == 0) {
            // the group's query rows, once per copy: box = the tokens' rows of this KV head, one dim half
            mbar_arrive_expect_tx(bar_q, (uint32_t)(COPIES * 2 * p.group_rows * 128));
#pragma unroll
            for (int c = 0; c < COPIES; ++c)
#pragma unroll
                for (int d = 0; d < 2; ++d)
                    tma_load_5d(base + d * QHALF + c * RPC * 128, &q_map, 0, 0, h, b * p.T + row0 / p.G, d, bar_q);
        }
        __syncwarp();
        for (int c = c0, w = 0; c < c1 && alive; c += kWinCols, w ^= 1) {
            window_wait();
            if (c + kWinCols < c1) window_request(win_u32 + (w ^ 1) * kWinBytes, lane, blk_row, slot_row, c + kWinCols + lane, c1);
            const int blk = win[w * (2 * kWinCols) + lane], slot = win[w * (2 * kWinCols) + kWinCols + lane];
            const bool ok = block_seen(blk, L);                      // (columns past c1 are -1)
            const unsigned got = __ballot_sync(0xffffffffu, ok);
            if (ok) queue[(tail + __popc(got & ((1u << lane) - 1u))) & (kTrQueue - 1)] = make_int2(blk, slot);
            tail += __popc(got);
            __syncwarp();
            while (alive && tail - head >= kAtTileCols) emit(kAtTileCols);
        }
        if (n_tree_blk > 0) {                                        // at most 3 + 4 entries are in the queue then
            if (lane < n_tree_blk) queue[(tail + lane) & (kTrQueue - 1)] = make_int2(kTreeTag + lane, 0);
            tail += n_tree_blk;
            __syncwarp();
        }
        while (alive && tail > head) emit(min(kAtTileCols, tail - head));
    } else if (warp == 1) {
        // ---------------------------------------------------------------- Q K^T issuer (the whole warp, converged)
        const uint32_t idesc = idesc_qk(MMA_M);
        const uint64_t k_desc0 = smem_desc_sw128_k(kv_u32, kImgGroup);
        bool alive = mbar_wait_warp(bar_q, 0, p.err, 50);
        int s = 0, sb = 0, s_old = 0;                                // stage and S buffer of tile i; stage of tile i - SBUFS
        uint32_t ph = 0, ph_old = 0;
        for (int i = 0; i < n_tiles && alive; ++i) {
            // the S buffer also held P of tile i - SBUFS: its P V must have completed
            if (i >= SBUFS) {
                alive = mbar_wait_warp(bar_empty(s_old), ph_old, p.err, 51);
                ph_old ^= (s_old + 1 == STAGES);
                s_old = (s_old + 1 == STAGES) ? 0 : s_old + 1;
            }
            alive = alive && mbar_wait_warp(bar_full(s), ph, p.err, 52);
            if (!alive) break;
            tc_fence_after();
            const uint64_t k_desc = k_desc0 + (uint64_t)((s * kAtStageBytes) >> 4);
#pragma unroll
            for (int g = 0; g < HALVES; ++g) {
                const uint64_t q_desc = smem_desc_sw128(base + g * 128 * 128);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    tc_mma_bf16(tmem_base + (uint32_t)((g * SBUFS + sb) * kAtTileKeys),
                                q_desc + (uint64_t)(((k >> 2) * QHALF + (k & 3) * 32) >> 4),
                                k_desc + (uint64_t)(((k >> 2) * kImgHalf + (k & 3) * 32) >> 4), idesc, k ? 1u : 0u);
                tc_commit(bar_s_full(g * SBUFS + sb));
            }
            ph ^= (s + 1 == STAGES);
            s = (s + 1 == STAGES) ? 0 : s + 1;
            sb = (sb + 1 == SBUFS) ? 0 : sb + 1;
        }
    } else if (warp == 2) {
        // ---------------------------------------------------------------- P V issuer (the whole warp, converged)
        const uint32_t idesc = idesc_pv(MMA_M);
        const uint64_t v_desc0 = smem_desc_sw128_mn(kv_u32 + kImgPart, kImgHalf, kImgGroup);
        bool alive = true;
        int s = 0, sb = 0;
        uint32_t ph_p = 0;
        for (int i = 0; i < n_tiles && alive; ++i) {
            const uint64_t v_desc = v_desc0 + (uint64_t)((s * kAtStageBytes) >> 4);
#pragma unroll
            for (int g = 0; g < HALVES && alive; ++g) {              // (set 0 has also zeroed the V rows that nobody may see)
                alive = mbar_wait_warp(bar_p_full(g * SBUFS + sb), ph_p, p.err, 53);
                if (!alive) break;
                tc_fence_after();
                issue_pv_tile(tmem_o + (uint32_t)((PAIR ? g : i % SETS) * kHeadDim),
                              tmem_base + (uint32_t)((g * SBUFS + sb) * kAtTileKeys), v_desc, idesc, i < SETS);
            }
            if (!alive) break;
            tc_commit(bar_empty(s));                                 // stage free, and O complete up to this tile
            s = (s + 1 == STAGES) ? 0 : s + 1;
            sb = (sb + 1 == SBUFS) ? 0 : sb + 1;
            ph_p ^= (sb == 0);
        }
    } else {
        // ---------------------------------------------------------------- softmax, one thread per MMA row
        const int set = SETS == 2 ? (warp - 3) >> 2 : 0;
        const int half = PAIR ? (warp - 3) >> 2 : 0;
        const int quarter = warp & 3;
        const int m_row = quarter * LANES + (lane % LANES);         // MMA row held by this tensor-memory lane
        const int copy = m_row / RPC, row = m_row % RPC + half * 128;       // which copy of the rows, which query row of the group
        const bool has_row = lane < LANES;
        const bool live_row = has_row && row < rows;
        const bool live_warp = (quarter * LANES) % RPC + half * 128 < rows;     // some lane of this warp holds a query row
        const unsigned long long sees = live_row ? anc[(row0 + row) / p.G] : 0ull;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const int worker = quarter * 32 + lane;                     // of the set's 128 threads
        float m_ref = -CUDART_INF_F, l_sum = 0.f;
        bool alive = true;
        int s = 0, s_prev = 0;                                      // ring stage of tile i and of this set's previous tile
        uint32_t ph = 0, ph_prev = 0;                               // parities of the "empty" phases that end those tiles
        int sb = set;                                               // S buffer of tile i (SETS < SBUFS)
        uint32_t ph_s = 0;
        ring_advance(s, ph, set, STAGES);
        const uint32_t my_o = tmem_o + (uint32_t)((set + half) * kHeadDim) + lane_base;   // this thread's O row
        for (int i = set; i < n_tiles && alive; i += SETS) {
            alive = mbar_wait(bar_s_full(half * SBUFS + sb), ph_s, p.err, 61);
            if (!alive) break;
            tc_fence_after();
            const int32_t *ids = tile_blk + s * kAtTileCols;
            const bool all_seen = plain[s] != 0;                    // four full history blocks: nothing to mask
            // V rows that nobody may see: history positions from seq_len on, padding nodes.  Thread -> (block, key, half).
            if (half == 0 && !all_seen) {
                const int c = worker >> 5, key = (worker >> 1) & 15, dims = worker & 1;
                const int blk = ids[c];
                const int valid = blk < kTreeTag ? L - blk * kBlock : n_nodes - (blk - kTreeTag) * kBlock;
                if (blk >= 0 && key >= valid) {
                    uint8_t *dst = kv_ptr + (size_t)s * kAtStageBytes + c * kEntryBytes + (key >> 3) * kImgGroup + dims * kImgHalf +
                                   kImgPart + (key & 7) * 128;
#pragma unroll
                    for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4 *>(dst + j * 16) = make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
            }
            const uint32_t s_tmem = tmem_base + lane_base + (uint32_t)((half * SBUFS + sb) * kAtTileKeys);
            if (live_warp) {
                float x[BPC * kBlock];
                {
                    uint32_t v[BPC][16];
#pragma unroll
                    for (int c = 0; c < BPC; ++c) tc_ld16_nowait(s_tmem + (copy * BPC + c) * 16, v[c]);
                    tc_wait_ld();
#pragma unroll
                    for (int c = 0; c < BPC; ++c)
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[c * 16 + e] = __uint_as_float(v[c][e]);
                }
                if (!all_seen) {
#pragma unroll
                    for (int c = 0; c < BPC; ++c) {                 // visible keys of each of this copy's blocks
                        const int blk = ids[copy * BPC + c];
                        uint32_t bits = 0xffffu;                    // lanes without a query row need no masking
                        if (live_row) {
                            if (blk < 0) bits = 0;
                            else if (blk < kTreeTag) bits = L - blk * kBlock < kBlock ? (1u << (L - blk * kBlock)) - 1u : 0xffffu;
                            else bits = (uint32_t)(sees >> ((blk - kTreeTag) * kBlock)) & 0xffffu;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (!((bits >> e) & 1u)) x[c * 16 + e] = -CUDART_INF_F;
                    }
                }
                alive = softmax_rest<COPIES>(x, s_tmem, my_o, copy, has_row, p.scale_log2, m_ref, l_sum, i >= SETS,
                                             // (the stage of this set's previous tile is released by the commit that follows
                                             // its P V; with at least four stages in the ring the parity is unambiguous)
                                             [&] { return mbar_wait(bar_empty(s_prev), ph_prev, p.err, 62); });
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p_full(half * SBUFS + sb));
            s_prev = s;
            ph_prev = ph;
            ring_advance(s, ph, SETS, STAGES);
#pragma unroll
            for (int k = 0; k < SETS; ++k) {
                sb = (sb + 1 == SBUFS) ? 0 : sb + 1;
                ph_s ^= (sb == 0);
            }
        }
        // ---- epilogue: merge the copies or sets, normalise, write out ----------------------------------------
        if (alive && n_tiles > 0)
            alive = mbar_wait(bar_empty((n_tiles - 1) % STAGES), ((n_tiles - 1) / STAGES) & 1, p.err, 63);
        tc_fence_after();
        const int mine = set * 128 + half * 128 + m_row;
        if (n_tiles > 0 && live_warp && alive) {
            float *dst = o_sm + mine * PITCH;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[2][16];
                tc_ld16_nowait(my_o + c * 32, v[0]);
                tc_ld16_nowait(my_o + c * 32 + 16, v[1]);
                tc_wait_ld();
                if (has_row) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        reinterpret_cast<uint4 *>(dst + c * 32)[e] = make_uint4(v[e >> 2][(e & 3) * 4], v[e >> 2][(e & 3) * 4 + 1],
                                                                                v[e >> 2][(e & 3) * 4 + 2], v[e >> 2][(e & 3) * 4 + 3]);
                }
            }
        }
        if (has_row) {
            m_sm[mine] = m_ref;
            l_sm[mine] = l_sum;
        }
        alive = softmax_warps_all<THREADS - 96>(alive);
        // A warp writes rows r0, r0 + WRITERS, ..: lane k works out row k's weights (the parts', normalised), place and
        // log-sum-exp, then the half-warps copy two rows at a time.
        const int r0 = warp - 3, n_mine = alive && rows > r0 ? (rows - r0 + WRITERS - 1) / WRITERS : 0;    // at most 32
        float w[PARTS];
        int orow = 0;
        if (lane < n_mine) {
            const int r = r0 + lane * WRITERS;
            float mx = -CUDART_INF_F, den = 0.f;
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
                w[c] = m_sm[c * RPC + r];
                mx = fmaxf(mx, w[c]);
            }
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
                w[c] = mx == -CUDART_INF_F ? 0.f : fast_exp2(w[c] - mx);
                den += w[c] * l_sm[c * RPC + r];
            }
            const float inv = den > 0.f ? 1.f / den : 0.f;
            const float lse2 = den > 0.f ? mx + log2f(den) : -CUDART_INF_F;
#pragma unroll
            for (int c = 0; c < PARTS; ++c) w[c] *= inv;
            const int tq = (row0 + r) / p.G, a = h * p.G + (row0 + r) % p.G;
            orow = CLUSTER || p.n_splits == 1 ? (b * p.T + tq) * p.Hq + a : blockIdx.x * p.group_rows + r;
            if (CLUSTER) row_lse[r] = lse2;
            else if (p.n_splits > 1) p.part_lse[orow] = lse2;
            else if (p.lse) p.lse[orow] = lse2 * kAtLn2;
        }
        const int side = lane >> 4, col = (lane & 15) * 4;          // four dims in either half of the row
#pragma unroll 4
        for (int k0 = 0; k0 < n_mine; k0 += 2) {
            const int k = min(k0 + side, n_mine - 1), r = r0 + k * WRITERS;          // (an odd last row is written twice)
            const long long o = __shfl_sync(0xffffffffu, orow, k);
            float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
            for (int c = 0; c < PARTS; ++c) {
                const float wc = __shfl_sync(0xffffffffu, w[c], k);
                const float *src = o_sm + (c * RPC + r) * PITCH + col;
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const float4 f = *reinterpret_cast<const float4 *>(src + 64 * d);
                    // (a part that saw no key, weight 0, may never have been written: its contents do not enter)
                    acc[d].x = wc != 0.f ? fmaf(wc, f.x, acc[d].x) : acc[d].x;
                    acc[d].y = wc != 0.f ? fmaf(wc, f.y, acc[d].y) : acc[d].y;
                    acc[d].z = wc != 0.f ? fmaf(wc, f.z, acc[d].z) : acc[d].z;
                    acc[d].w = wc != 0.f ? fmaf(wc, f.w, acc[d].w) : acc[d].w;
                }
            }
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                if (CLUSTER) {                                       // in place of the row's first part, for the cluster's merge
                    if (k0 + side < n_mine) *reinterpret_cast<float4 *>(o_sm + r * PITCH + col + 64 * d) = acc[d];
                } else if (p.n_splits == 1)
                    *reinterpret_cast<uint2 *>(p.out + (o * kHeadDim + col + 64 * d) * 2) =
                        make_uint2(pack_bf16x2(acc[d].x, acc[d].y), pack_bf16x2(acc[d].z, acc[d].w));
                else
                    *reinterpret_cast<float4 *>(p.part_o + o * kHeadDim + col + 64 * d) = acc[d];
            }
        }
    }

    if constexpr (CLUSTER) {
        // ---- the cluster's merge: block `split` writes rows split, split + n_splits, ..  A warp takes four, two or one row at a
        // time, so that eight reads are in flight whatever the size of the cluster: read e belongs to row e >> lg and block
        // e & (per - 1), and lane e holds its weight.
        cluster_barrier();
        if (warp >= 3) {
            const int lg = p.n_splits <= 2 ? 1 : p.n_splits <= 4 ? 2 : 3, per = 1 << lg, step = p.n_splits * WRITERS;
#pragma unroll 1
            for (int r0 = split + p.n_splits * (warp - 3); r0 < rows; r0 += step * (kTrMaxCluster >> lg)) {
                const int my_r = r0 + (lane >> lg) * step, my_q = lane & (per - 1);
                const bool mine = lane < kTrMaxCluster && my_r < rows && my_q < p.n_splits;
                const float lse2 = mine ? ld_cluster(at_rank(row_lse + my_r, (uint32_t)my_q)) : -CUDART_INF_F;
                float4 f[kTrMaxCluster];
#pragma unroll
                for (int e = 0; e < kTrMaxCluster; ++e) {
                    const int r = r0 + (e >> lg) * step, q = e & (per - 1);
                    f[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (r < rows && q < p.n_splits) f[e] = ld_cluster4(at_rank(o_sm + r * PITCH + lane * 4, (uint32_t)q));
                }
                float mx = lse2;
                for (int o = per >> 1; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                float w = lse2 == -CUDART_INF_F ? 0.f : fast_exp2(lse2 - mx), den = w;
                for (int o = per >> 1; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
                w *= den > 0.f ? 1.f / den : 0.f;
                const int tq = (row0 + my_r) / p.G, a = h * p.G + (row0 + my_r) % p.G;
                const long long my_row = ((long long)b * p.T + tq) * p.Hq + a;
                if (p.lse && mine && my_q == 0) p.lse[my_row] = den > 0.f ? (mx + log2f(den)) * kAtLn2 : -CUDART_INF_F;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int e = 0; e < kTrMaxCluster; ++e) {            // (places of no row or block have no weight)
                    const float we = __shfl_sync(0xffffffffu, w, e);
                    acc.x = we != 0.f ? fmaf(we, f[e].x, acc.x) : acc.x;
                    acc.y = we != 0.f ? fmaf(we, f[e].y, acc.y) : acc.y;
                    acc.z = we != 0.f ? fmaf(we, f[e].z, acc.z) : acc.z;
                    acc.w = we != 0.f ? fmaf(we, f[e].w, acc.w) : acc.w;
                    if ((e & (per - 1)) == per - 1) {                // the row's last
                        const long long orow = __shfl_sync(0xffffffffu, my_row, e);
                        if (r0 + (e >> lg) * step < rows)
                            reinterpret_cast<uint2 *>(p.out + orow * kHeadDim * 2)[lane] =
                                make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
                        acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                }
            }
        }
        cluster_barrier();                                           // nobody leaves while its shared memory is read
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)kAtTmemCols)
                     : "memory");
    }
}

// Merges the splits of one query row: out = sum_s w_s o_s / sum_s w_s with w_s = 2^(lse_s - max lse).  One warp per row,
// four output dims per thread, the loads of four splits in flight at a time.
__global__ void __launch_bounds__(256)
tree_combine_kernel(const TreeAttnParams p, int total)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int wi = 8 * blockIdx.x + (threadIdx.x >> 5);
    if (wi >= total) return;
    const int row = wi % p.R, bh = wi / p.R;
    const int b = bh / p.Hkv, h = bh % p.Hkv;
    const int tq = row / p.G, a = h * p.G + row % p.G;
    if (tq >= p.n_nodes[b]) return;
    const int grp = row / p.group_rows, r = row % p.group_rows;
    const long long prow0 = ((long long)bh * p.n_splits * p.n_groups + grp) * p.group_rows + r;    // partial row of split 0
    const long long pstride = (long long)p.n_groups * p.group_rows;
    float mx = -CUDART_INF_F;
    for (int s = lane; s < p.n_splits; s += 32) mx = fmaxf(mx, p.part_lse[prow0 + s * pstride]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float den = 0.f;
    if (mx > -CUDART_INF_F) {
#pragma unroll 1
        for (int s0 = 0; s0 < p.n_splits; s0 += 4) {
            float w[4];
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const bool in = s0 + u < p.n_splits;
                const long long prow = prow0 + (in ? s0 + u : s0) * pstride;
                w[u] = in ? p.part_lse[prow] : -CUDART_INF_F;
                v[u] = reinterpret_cast<const float4 *>(p.part_o + prow * kHeadDim)[lane];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float ws = fast_exp2(w[u] - mx);               // 0 for the splits past the last one
                acc.x += ws * v[u].x; acc.y += ws * v[u].y; acc.z += ws * v[u].z; acc.w += ws * v[u].w;
                den += ws;
            }
        }
    }
    const bool any = den > 0.f;                                      // some split saw a key
    if (!any) den = 1.f;
    const long long orow = ((long long)b * p.T + tq) * p.Hq + a;
    reinterpret_cast<uint2 *>(p.out + orow * kHeadDim * 2)[lane] =
        make_uint2(pack_bf16x2(acc.x / den, acc.y / den), pack_bf16x2(acc.z / den, acc.w / den));
    if (p.lse && lane == 0) p.lse[orow] = any ? (mx + log2f(den)) * kAtLn2 : -CUDART_INF_F;
}

// ---- host side -----------------------------------------------------------------------------------------
struct TreePlan {
    int n_groups, group_rows, n_splits, cols_per_split;
    bool in_cluster;
    long long items;
    size_t workspace;
};

static TreePlan tree_plan(const oasis_dims_t *dims, int T, int n_cols)
{
    TreePlan pl;
    const int G = dims->n_q_heads / dims->n_kv_heads, most_tokens = 256 / G;
    pl.n_groups = (T + most_tokens - 1) / most_tokens;
    pl.group_rows = (T + pl.n_groups - 1) / pl.n_groups * G;         // whole nodes, as evenly as they go
    // all thread blocks resident at once (one per SM) as far as the column list can be split, eight columns per split
    const long long items = (long long)dims->batch * dims->n_kv_heads * pl.n_groups;
    long long s = items > 0 ? sm_count() / items : 1;
    const long long most = (n_cols + 7) / 8;
    if (s > most) s = most;
    if (s < 1) s = 1;
    // The splits of a row are a cluster of two, three, four or eight thread blocks, which merges them through distributed shared
    // memory, where as many clusters as are needed run at once, a coarser split costs no more than a few tiles of four
    // columns against the finest one, and the rows are few or the blocks many; else the partials go through the workspace and a
    // second launch.  In a graph, 32 query and 8 KV heads, 5 / 16 / 64 nodes, cluster against workspace:
    //   1 request  x  18 columns   8.4 / 10.7 / 16.5   9.4 /  9.6 / 12.9 us   (the second launch spreads over idle SMs)
    //   4 requests x 130 columns  13.8 / 15.2 / 24.4  16.7 / 17.0 / 25.4 us
    //   5 requests x  62 columns  12.2 / 13.2 / 21.7  13.4 / 13.4 / 23.5 us
    //   8 requests x 130 columns, 32 nodes      22.1                25.9 us
    // Launched one by one, the cluster also saves the host 2 us a call.  Clusters of five (2 x 35 columns, 64 nodes) take 20 us
    // against 15.6.  A tile more takes 0.5 us, with two MMAs per tile 1 us, and the second launch 2 to 3: seven ragged requests
    // of 302 columns in fours instead of five splits (three tiles more) 21.3 against 22.3, 3 x 130 columns in fours instead of six
    // (three more) 12.7 / 14.2 / 23.4 against 13.7 / 14.7 / 23.1.
    const long long more_tiles = pl.group_rows <= 128 ? 4 : 2;
    long long c = s >= kTrMaxCluster ? kTrMaxCluster : s < 4 ? s : 4;
    while (c > 1 && clusters_at_once((int)c) < items) c = c == kTrMaxCluster ? 4 : c - 1;
    pl.in_cluster = c > 1 && n_cols / (4 * c) <= n_cols / (4 * s) + more_tiles && (pl.group_rows <= 32 || 2 * items * c >= sm_count());
    if (pl.in_cluster) s = c;
    pl.cols_per_split = (int)((n_cols + s - 1) / s);
    pl.n_splits = (n_cols + pl.cols_per_split - 1) / pl.cols_per_split;
    if (pl.n_splits == 1) pl.in_cluster = false;
    pl.items = items * pl.n_splits;
    pl.workspace = pl.n_splits > 1 && !pl.in_cluster ? (size_t)pl.items * pl.group_rows * (kHeadDim + 1) * sizeof(float) : 0;
    return pl;
}

static int check_tree(const oasis_dims_t *dims, int T, int n_cols, const char *who)
{
    if (int rc = check_dims(dims)) return rc;
    if (T < 1 || T > OASIS_MAX_TREE)
        return fail(OASIS_ERR_INVALID_ARG, "%s: n_tree %d outside [1, %d]", who, T, OASIS_MAX_TREE);
    if (n_cols < 1 || n_cols > (1 << 26)) return fail(OASIS_ERR_INVALID_ARG, "%s: n_cols %d", who, n_cols);
    const int G = dims->n_q_heads / dims->n_kv_heads;
    if (G > 128) return fail(OASIS_ERR_UNSUPPORTED, "%s: %d query heads per KV head > 128", who, G);
    if ((long long)dims->batch * dims->n_kv_heads * T * G > 0x7fffffffLL)
        return fail(OASIS_ERR_UNSUPPORTED, "%s: more than 2^31 query rows", who);
    return OASIS_OK;
}

}  // namespace oasis

extern "C" size_t oasis_tree_attn_workspace_bytes(const oasis_dims_t *dims, int32_t n_tree, int32_t n_cols)
{
    using namespace oasis;
    if (check_tree(dims, n_tree, n_cols, "oasis_tree_attn_workspace_bytes") != OASIS_OK) return 0;
    return tree_plan(dims, n_tree, n_cols).workspace;
}

extern "C" int oasis_tree_attn(const oasis_dims_t *dims, const void *q, int32_t n_tree, const void *tree_kv,
                               const int32_t *parent, const int32_t *n_nodes, const void *hbm_pool,
                               const int32_t *slot_tbl, const int32_t *blk_tbl, int32_t n_cols, const int32_t *seq_len,
                               float scale, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace oasis;
    const char *who = "oasis_tree_attn";
    if (int rc = check_tree(dims, n_tree, n_cols, who)) return rc;
    if (!(scale > 0.f) || scale > 3.0e38f) return fail(OASIS_ERR_INVALID_ARG, "%s: scale %g", who, (double)scale);
    if (dims->batch == 0) return OASIS_OK;
    if (!q || !tree_kv || !parent || !n_nodes || !hbm_pool || !slot_tbl || !blk_tbl || !seq_len || !out)
        return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    if (!aligned16(q) || !aligned16(tree_kv) || !aligned16(hbm_pool) || !aligned16(out))
        return fail(OASIS_ERR_INVALID_ARG, "%s: q, tree_kv, hbm_pool and out must be 16-byte aligned", who);
    const TreePlan pl = tree_plan(dims, n_tree, n_cols);
    if (pl.workspace > 0) {
        if (!workspace || workspace_bytes < pl.workspace)
            return fail(OASIS_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", who, pl.workspace,
                        workspace ? workspace_bytes : (size_t)0);
        if (!aligned16(workspace)) return fail(OASIS_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", who);
    }
    if (pl.items * pl.group_rows > 0x7fffffffLL) return fail(OASIS_ERR_UNSUPPORTED, "%s: grid too large", who);
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return fail(OASIS_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available", who);

    // The pool as attn_tc.cu sees it: one box = one 8 KiB entry, landing as [group][half][K, V][8 rows][128 B].
    CUtensorMap pool_map, tree_map, q_map;
    const cuuint64_t pool_parts = (kBoundsCheck && bounds().n_slots < (1ll << 30)) ? (cuuint64_t)(2 * bounds().n_slots) : (cuuint64_t)1 << 31;
    const cuuint64_t pdim[5] = {64, 8, pool_parts, 2, 2}, pstride[4] = {256, 4096, 128, 2048};
    const cuuint32_t pbox[5] = {64, 8, 2, 2, 2}, estr[5] = {1, 1, 1, 1, 1};
    CUresult cr = encode(&pool_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(hbm_pool), pdim, pstride, pbox, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (cr != CUDA_SUCCESS) return fail(OASIS_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed (%d)", who, (int)cr);
    // The tree buffer [B][T][Hkv][K, V][2 x 64 dims], innermost first: 64 elements | nodes | (head, part) | dim half |
    // request.  One box = 8 nodes of one head, landing as [half][K, V][8 rows][128 B] = one row group of a block image;
    // nodes past T read as zero.
    const cuuint64_t Hkv = (cuuint64_t)dims->n_kv_heads, T64 = (cuuint64_t)n_tree;
    const cuuint64_t tdim[5] = {64, T64, 2 * Hkv, 2, (cuuint64_t)dims->batch}, tstride[4] = {Hkv * 512, 256, 128, T64 * Hkv * 512};
    const cuuint32_t tbox[5] = {64, 8, 2, 2, 1};
    cr = encode(&tree_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(tree_kv), tdim, tstride, tbox, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (cr != CUDA_SUCCESS) return fail(OASIS_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed (%d)", who, (int)cr);
    // The queries [B * T][Hkv][G][2 x 64 dims], innermost first: 64 elements | head of the group | KV head | token | dim half.
    // One box = the query rows of one row group, one dim half, 128 bytes per row in the order (token, head of the group).
    const cuuint64_t G64 = (cuuint64_t)(dims->n_q_heads / dims->n_kv_heads), Hq64 = (cuuint64_t)dims->n_q_heads;
    const cuuint64_t qdim[5] = {64, G64, Hkv, (cuuint64_t)dims->batch * T64, 2}, qstride[4] = {256, G64 * 256, Hq64 * 256, 128};
    const cuuint32_t qbox[5] = {64, (cuuint32_t)G64, 1, (cuuint32_t)(pl.group_rows / (int)G64), 1};
    cr = encode(&q_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(q), qdim, qstride, qbox, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (cr != CUDA_SUCCESS) return fail(OASIS_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed (%d)", who, (int)cr);

    TreeAttnParams p = {};
    p.slot_tbl = slot_tbl; p.blk_tbl = blk_tbl; p.seq_len = seq_len; p.parent = parent;
    p.n_nodes = n_nodes; p.out = (uint8_t *)out; p.lse = lse; p.err = error_word();
    p.scale_log2 = scale * kAtLog2e;
    p.T = n_tree; p.Hq = dims->n_q_heads; p.Hkv = dims->n_kv_heads; p.G = p.Hq / p.Hkv; p.n_cols = n_cols; p.R = n_tree * p.G;
    p.n_splits = pl.n_splits; p.cols_per_split = pl.cols_per_split; p.n_groups = pl.n_groups; p.group_rows = pl.group_rows;
    p.n_slots = bounds().n_slots;
    if (pl.n_splits > 1 && !pl.in_cluster) {
        p.part_o = (float *)workspace;
        p.part_lse = p.part_o + (size_t)pl.items * pl.group_rows * kHeadDim;
    }
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)pl.n_splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pl.items);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = pl.in_cluster ? 2 : 1;
#define OASIS_TREE_LAUNCH_AS(M, C, P, X)                                                                                      \
    do {                                                                                                                      \
        e = allow_dynamic_shared(reinterpret_cast<const void *>(tree_attn_tc_kernel<M, C, P, X>), tr_smem(M, P));              \
        if (e == cudaSuccess) prefer_max_shared_carveout(tree_attn_tc_kernel<M, C, P, X>);                                    \
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, tree_attn_tc_kernel<M, C, P, X>, pool_map, tree_map, q_map, p);    \
    } while (0)
#define OASIS_TREE_LAUNCH(M, C, P)                                                                                            \
    do {                                                                                                                      \
        cfg.blockDim = dim3(tr_threads(M, C, P));                                                                             \
        cfg.dynamicSmemBytes = tr_smem(M, P);                                                                                 \
        if (pl.in_cluster) OASIS_TREE_LAUNCH_AS(M, C, P, true);                                                               \
        else OASIS_TREE_LAUNCH_AS(M, C, P, false);                                                                            \
    } while (0)
    if (pl.group_rows <= 16) OASIS_TREE_LAUNCH(64, 4, false);       // four copies of <= 16 rows, one block of a tile each
    else if (pl.group_rows <= 32) OASIS_TREE_LAUNCH(64, 2, false);  // two copies of <= 32 rows, two blocks each
    else if (pl.group_rows <= 64) OASIS_TREE_LAUNCH(128, 2, false); // two copies of <= 64 rows: half the softmax work per thread
    else if (pl.group_rows <= 128) OASIS_TREE_LAUNCH(128, 1, false);   // two softmax warp sets, alternate tiles
    else OASIS_TREE_LAUNCH(128, 1, true);                           // two softmax warp sets, 128 rows each
#undef OASIS_TREE_LAUNCH
#undef OASIS_TREE_LAUNCH_AS
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    if (pl.n_splits > 1 && !pl.in_cluster) {
        // (the merge's thread blocks become resident while the attention still runs and wait there for the partials)
        const int total = dims->batch * p.Hkv * p.R;
        cfg.gridDim = dim3((unsigned)((total + 7) / 8));
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        cfg.numAttrs = 1;
        prefer_max_shared_carveout(tree_combine_kernel);
        e = cudaLaunchKernelEx(&cfg, tree_combine_kernel, p, total);
        if (e != cudaSuccess) return fail(OASIS_ERR_CUDA, "%s: combine launch: %s", who, cudaGetErrorString(e));
        return check_launch(who);
    }
    return OASIS_OK;
}
