// Attention over a working set held in 4 bits (packed.cuh), with the local window in bf16, on the 5th-generation tensor cores.
//
// Work item = (request, KV head, row group, split of the columns), one thread block of 128 threads.  Tiles of eight 16-token blocks.
// Other than in the bf16 kernels the keys and values, which have to pass through registers anyway, are the A operands in tensor
// memory, and the query rows the columns:
//   S[token][row] = K Q^T    thread = token: 64 B of codes become the token's 128 bf16 dims, 64 columns of its tensor-memory lane
//   O[dim][row]  += V^T P    thread = dim: 8 B of codes per block become the dim's 16 tokens, 8 columns of its lane
// Q (K-major) and P (row-major by token) are the B operands in shared memory.  So 4-bit data crosses shared memory once, bf16 data
// never (as bf16 tiles in shared memory they would be written and read there, 2.5 times the time that HBM takes to bring them).
// A row's logits lie across the threads: the reference maximum that its weights are taken against is shared and raised only when a
// logit exceeds it by 2^8, which one vote per tile finds out; the rows' sums are kept per thread and added up at the end.
// One tile after the other in a thread block: wait for its entries, keys, K Q^T, (meanwhile) values, softmax, V^T P (meanwhile the
// next keys).  Four thread blocks per SM (two with more than 32 rows) overlap each other's waits.
// Entries come as bulk copies, one per block, a ring of two to four tiles ahead.  Columns that no row sees are left out when the
// column list of the split is read (compacted in order: the result does not depend on the launch).  The local columns, at most one
// tile, are the first tile of split 0, read straight from global memory while the ring fills.
// Rows: up to 64 per thread block (16, 32 or 64 columns of the products); more are cut into row groups.
// Splits of a row merge inside a thread-block cluster where eight reach, else through the workspace and a second launch.
// Precision: (c - 8) s is exact in bf16; logits, maxima, sums and accumulators are fp32; the weights go to V^T P as bf16 (half a
// step, 2^-8 of a weight), because both operands of one tcgen05.mma kind::f16 have the same type; the sum that divides them is of
// the unrounded ones.
#include <cuda.h>
#include <math_constants.h>

#include "packed.cuh"
#include "tc_common.cuh"

namespace oasis {

constexpr int kPaTileCols = 8, kPaTileKeys = kPaTileCols * kBlock;       // 128 tokens: the rows of one MMA
constexpr int kPaStageBytes = kPaTileCols * kPackedBytes;                // 18 KiB
constexpr int kPaListCols = 256;                                         // columns of a split at most
constexpr int kPaThreads = 128;
constexpr int kPaMaxCluster = 8;
__host__ __device__ constexpr int pa_blocks(int n) { return n <= 32 ? 4 : 2; }              // thread blocks per SM
__host__ __device__ constexpr int pa_stages(int n) { return n <= 32 ? 2 : 4; }
__host__ __device__ constexpr int pa_tmem_cols(int n) { return n <= 32 ? 128 : 256; }       // K, V: 64 (shared up to 32 rows); S, O: n each
// Shared memory: Q [dim half][n rows][128 B] | P [128 tokens][2 n B] | ring | column list | statistics and barriers.
constexpr int kPaMisc = 1536;
__host__ __device__ constexpr int pa_smem(int n)
{
    return 1024 + n * kRowBytes + kPaTileKeys * 2 * n + pa_stages(n) * kPaStageBytes + kPaListCols * 8 + (n <= 32 ? 768 : kPaMisc);
}
static_assert((pa_smem(16) + 1024) * 4 <= 233472 && (pa_smem(32) + 1024) * 4 <= 233472 && (pa_smem(64) + 1024) * 2 <= 233472, "thread blocks per SM");
static_assert(pa_stages(32) * kPaStageBytes >= 32 * kHeadDim * 4 && pa_stages(64) * kPaStageBytes >= 64 * kHeadDim * 4, "the accumulator fits into the ring");

struct PackedAttnParams {
    const uint8_t *q, *packed, *local;
    const int32_t *slot_tbl, *blk_tbl, *seq_len;
    uint8_t *out;
    float *lse;
    float *part_o;      // [items][rows per group][128] fp32, normalised (runs through the workspace only)
    float *part_lse;    // [items][rows per group]      log2 domain
    int32_t *err;
    float scale_log2;
    int T, Hq, Hkv, G, n_cols, local_col, R, n_splits, tiles_per_split, n_groups, group_rows;
    Bounds bd;
};

__device__ __forceinline__ uint32_t pa_at_rank(const void *place, uint32_t rank)
{
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(place)), "r"(rank));
    return addr;
}
__device__ __forceinline__ float pa_ld_cluster(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 pa_ld_cluster4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// fp32 <-> integers of the same order (for the integer maximum over a warp).
__device__ __forceinline__ int ordered(float f)
{
    const int b = __float_as_int(f);
    return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b ^ ((b >> 31) & 0x7fffffff)); }

// Instruction descriptors (kind::f16, fp32 accumulator, bf16 operands, M = 128).
__device__ __forceinline__ uint32_t pa_idesc(int n, bool b_mn_major)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn_major ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// P: rows = tokens of 2 N bytes, swizzled over as many bytes (16 rows: 32, 32 rows: 64, 64 rows: 128), groups of eight tokens.
template <int N>
__device__ __forceinline__ uint64_t pa_p_desc(uint32_t addr)
{
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3ffffu) >> 4);
    d |= (uint64_t)1 << 16;                                              // (one atom holds all columns)
    d |= (uint64_t)((16 * N) >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)(N == 64 ? 2 : N == 32 ? 4 : 6) << 61;
    return d;
}
template <int N>
__device__ __forceinline__ uint32_t pa_p_chunk(int token, int c)         // byte offset of columns 8 c .. 8 c + 7 of a token's row
{
    const int x = N == 64 ? token & 7 : N == 32 ? (token >> 1) & 3 : (token >> 2) & 1;
    return (uint32_t)(token * 2 * N + ((c ^ x) << 4));
}

// N: columns of the products (query rows, padded).
template <int N, bool CLUSTER>
__global__ void __launch_bounds__(kPaThreads, pa_blocks(N))
packed_attn_kernel(const PackedAttnParams p)
{
    constexpr int STAGES = pa_stages(N);
    constexpr bool SHARED_KV = N <= 32;                     // keys and values take turns in the same 64 columns of tensor memory
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    uint8_t *const p_ptr = base_ptr + N * kRowBytes;
    uint8_t *const ring = p_ptr + kPaTileKeys * 2 * N;
    int2 *const list = reinterpret_cast<int2 *>(ring + STAGES * kPaStageBytes);           // (block, slot)
    float *const neg_m = reinterpret_cast<float *>(list + kPaListCols);                     // [N] minus the rows' reference maxima
    float *const l_sm = neg_m + N;                                                          // [N]; while a maximum is raised: factors
    uint64_t *const bars = reinterpret_cast<uint64_t *>(l_sm + N);
    int2 *const s_local = reinterpret_cast<int2 *>(bars + STAGES + 2);                      // [8] the local columns
    int *const s_cnt = reinterpret_cast<int *>(s_local + kPaTileCols);                      // [8]
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(s_cnt + 8);
    volatile int *const dead = reinterpret_cast<int *>(tmem_slot + 1);
    const uint32_t bar0 = smem_u32(bars), bar_s = bar0 + 8u * STAGES, bar_o = bar_s + 8u;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int grp = CLUSTER ? (blockIdx.x / p.n_splits) % p.n_groups : blockIdx.x % p.n_groups;
    const int split = CLUSTER ? blockIdx.x % p.n_splits : (blockIdx.x / p.n_groups) % p.n_splits;
    const int bh = blockIdx.x / (p.n_groups * p.n_splits);
    const int b = bh / p.Hkv, h = bh % p.Hkv;
    const int row0 = grp * p.group_rows, rows = min(p.group_rows, p.R - row0);
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)pa_tmem_cols(N)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < STAGES + 2; ++s) mbar_init(bar0 + 8u * s, 1);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < N) neg_m[tid] = CUDART_INF_F;
    // This launch may have been brought onto the SMs before the previous one ended: what that wrote is read from here on.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- the split's columns ------------------------------------------------------------------------------------
    // Tiles of a row: the local columns (if any), then eight packed columns each.
    const int has_local = p.n_cols > p.local_col;
    const int t0 = split * p.tiles_per_split, t1 = t0 + p.tiles_per_split;
    const int c0 = max(t0 - has_local, 0) * kPaTileCols, c1 = min((t1 - has_local) * kPaTileCols, p.local_col);
    const int32_t *blk_row = p.blk_tbl + (long long)bh * p.n_cols, *slot_row = p.slot_tbl + (long long)bh * p.n_cols;
    const long long L = p.seq_len[b], last = L + p.T - 1;               // last position that a row sees
    int2 col[2];
    unsigned got[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = c0 + tid + 128 * k;
        col[k] = make_int2(-1, -1);
        if (c < c1) col[k] = make_int2(blk_row[c], slot_row[c]);
    }
    int2 near = make_int2(-1, -1);
    if (tid < kPaTileCols && has_local && t0 == 0 && p.local_col + tid < p.n_cols)
        near = make_int2(blk_row[p.local_col + tid], slot_row[p.local_col + tid]);
    // Q: 16 bytes (chunk c of row r) at a time; rows past the group's are zero
#pragma unroll 4
    for (int i = tid; i < N * 16; i += kPaThreads) {
        const int r = i >> 4, c = i & 15;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const int tq = (row0 + r) / p.G, a = h * p.G + (row0 + r) % p.G;
            v = *reinterpret_cast<const uint4 *>(p.q + (((long long)b * p.T + tq) * p.Hq + a) * kRowBytes + c * 16);
        }
        *reinterpret_cast<uint4 *>(base_ptr + (c >> 3) * (N * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        bool ok = col[k].x >= 0 && (long long)col[k].x * kBlock <= last;
        if (kBoundsCheck && ok) ok = in_range(col[k].y, p.bd.n_slots, p.bd, kErrSlot);
        got[k] = __ballot_sync(0xffffffffu, ok);
        if (lane == 0) s_cnt[k * 4 + warp] = __popc(got[k]);
    }
    if (warp == 0) {
        bool ok = near.x >= 0 && (long long)near.x * kBlock <= last;
        if (kBoundsCheck && ok) ok = in_range(near.y, p.bd.n_slots, p.bd, kErrSlot);
        if (lane < kPaTileCols) s_local[lane] = ok ? near : make_int2(-1, -1);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    int count = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w == warp && ((got[k] >> lane) & 1u)) list[count + __popc(got[k] & ((1u << lane) - 1u))] = col[k];
            count += s_cnt[k * 4 + w];
        }
    int do_local = 0;
#pragma unroll
    for (int k = 0; k < kPaTileCols; ++k) do_local |= s_local[k].x >= 0;
    const int packed_tiles = (count + kPaTileCols - 1) / kPaTileCols, n_tiles = do_local + packed_tiles;
    const uint32_t tmem = *tmem_slot, lane_base = (uint32_t)(warp * 32) << 16;
    const uint32_t t_k = tmem, t_v = tmem + (SHARED_KV ? 0 : 64), t_s = t_v + 64, t_o = t_s + N;
    __syncthreads();                                                     // the list is complete

    // Warp 0, lanes 0..7: one entry each of packed tile `pi` into its stage.
    auto request = [&](int pi) {
        const int n = min(kPaTileCols, count - pi * kPaTileCols), s = pi % STAGES;
        if (lane == 0) mbar_arrive_expect_tx(bar_full(s), (uint32_t)(n * kPackedBytes));
        __syncwarp();
        if (lane < n)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_u32(ring) + (uint32_t)(s * kPaStageBytes + lane * kPackedBytes)),
                           "l"(p.packed + (long long)list[pi * kPaTileCols + lane].y * kPackedBytes), "r"((uint32_t)kPackedBytes),
                           "r"(bar_full(s)) : "memory");
        __syncwarp();
    };
    if (warp == 0)
        for (int pi = 0; pi < min(STAGES, packed_tiles); ++pi) request(pi);

    float l[N];
#pragma unroll
    for (int n = 0; n < N; ++n) l[n] = 0.f;
    const int kb = 2 * warp + (lane >> 4), tok = lane & 15;             // this thread's block of the tile and token, for the keys
    int issued = min(STAGES, packed_tiles), done_tiles = 0;
#pragma unroll 1
    for (int i = 0; i < n_tiles; ++i) {
        const bool loc = do_local && i == 0;
        const int pi = i - do_local, s = pi % STAGES;
        const uint8_t *const stage = ring + s * kPaStageBytes;
        const int2 mine = loc ? s_local[kb] : pi * kPaTileCols + kb < count ? list[pi * kPaTileCols + kb] : make_int2(-1, -1);
        // the first column (query row) that sees this thread's token
        const long long ahead = (long long)mine.x * kBlock + tok - L;
        const int n_min = mine.x < 0 || ahead >= p.T ? N : ahead <= 0 ? 0 : min(max((int)ahead * p.G - row0, 0), N);
        // ---- keys
        uint32_t r[64];
        if (loc) {
#pragma unroll
            for (int e = 0; e < 64; ++e) r[e] = 0;
            if (n_min < N) {
                const uint4 *src = reinterpret_cast<const uint4 *>(p.local + (long long)mine.y * kEntryBytes + tok * kRowBytes);
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const uint4 v = src[c];
                    r[4 * c] = v.x; r[4 * c + 1] = v.y; r[4 * c + 2] = v.z; r[4 * c + 3] = v.w;
                }
            }
        } else {
            if (!mbar_wait(bar_full(s), (pi / STAGES) & 1, p.err, 81)) *dead = 1;
            const uint8_t *ent = stage + kb * kPackedBytes;
            const uint2 sc = *reinterpret_cast<const uint2 *>(ent + kPackedKScale + tok * 8);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 w = *reinterpret_cast<const uint4 *>(ent + c * 256 + tok * 16);
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int byte = 2 * c + g;
                    uint32_t s2, c2;
                    scale_pair(__byte_perm(byte < 4 ? sc.x : sc.y, 0u, 0x4040 | (byte & 3) | ((byte & 3) << 8)), s2, c2);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t o[4];
                        dequant_word(ww[2 * g + e], s2, c2, o);
#pragma unroll
                        for (int k = 0; k < 4; ++k) r[16 * c + 8 * g + 4 * e + k] = o[k];
                    }
                }
            }
        }
        // V^T P of the previous tile has read its values and weights, and O is complete up to it
        if (i > 0 && !mbar_wait(bar_o, (i - 1) & 1, p.err, 82)) *dead = 1;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_st16(t_k + lane_base + c * 16, *reinterpret_cast<const uint32_t(*)[16]>(r + 16 * c));
        tc_wait_st();
        tc_fence_before();
        __syncthreads();
        if (*dead) break;
        if (warp == 0) {
            tc_fence_after();
            const uint64_t q_desc = smem_desc_sw128(base);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                tc_mma_bf16_ts(t_s, t_k + 8 * k, q_desc + (uint64_t)(((k >> 2) * (N * 128) + (k & 3) * 32) >> 4), pa_idesc(N, false), k ? 1u : 0u);
            tc_commit(bar_s);
        }
        // ---- values: thread = dim
        if (loc) {
#pragma unroll
            for (int k = 0; k < kPaTileCols; ++k) {
                const int2 e = s_local[k];
#pragma unroll
                for (int j = 0; j < 8; ++j) r[8 * k + j] = 0;
                if (e.x >= 0) {                                          // (tokens past the last visible one may hold anything)
                    const uint16_t *src = reinterpret_cast<const uint16_t *>(p.local + (long long)e.y * kEntryBytes + kPartBytes) + tid;
                    const int n = (int)min((long long)kBlock, last - (long long)e.x * kBlock + 1);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t lo = 2 * j < n ? src[2 * j * kHeadDim] : 0u, hi = 2 * j + 1 < n ? src[(2 * j + 1) * kHeadDim] : 0u;
                        r[8 * k + j] = lo | hi << 16;
                    }
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPaTileCols; ++k) {
                const uint8_t *ent = stage + k * kPackedBytes;
                const uint2 w = *reinterpret_cast<const uint2 *>(ent + kPackedV + tid * 8);
                uint32_t s2, c2, o[4];
                scale_pair(ent[kPackedVScale + tid] * 0x00010001u, s2, c2);
                dequant_word(w.x, s2, c2, o);
#pragma unroll
                for (int j = 0; j < 4; ++j) r[8 * k + j] = o[j];
                dequant_word(w.y, s2, c2, o);
#pragma unroll
                for (int j = 0; j < 4; ++j) r[8 * k + 4 + j] = o[j];
            }
        }
        if (!mbar_wait(bar_s, i & 1, p.err, 83)) *dead = 1;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_st16(t_v + lane_base + c * 16, *reinterpret_cast<const uint32_t(*)[16]>(r + 16 * c));
        // ---- softmax: thread = token, one logit per query row
        float x[N];
        {
            uint32_t v[N / 16][16];
#pragma unroll
            for (int c = 0; c < N / 16; ++c) tc_ld16_nowait(t_s + lane_base + c * 16, v[c]);
            tc_wait_ld();
#pragma unroll
            for (int n = 0; n < N; ++n) x[n] = __uint_as_float(v[n >> 4][n & 15]);
        }
        tc_wait_st();
        const bool masked = __any_sync(0xffffffffu, n_min > 0);
        if (masked) {
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (n < n_min) x[n] = -CUDART_INF_F;
        }
        float top = -CUDART_INF_F;
#pragma unroll
        for (int n = 0; n < N; n += 4) {
            const float4 m = *reinterpret_cast<const float4 *>(neg_m + n);
            top = max3(top, fmaf(x[n], p.scale_log2, m.x), fmaf(x[n + 1], p.scale_log2, m.y));
            top = max3(top, fmaf(x[n + 2], p.scale_log2, m.z), fmaf(x[n + 3], p.scale_log2, m.w));
        }
        const int raise = __syncthreads_or(top > 8.f);                   // (also: every thread has read the stage)
        if (*dead) break;
        if (!loc) ++done_tiles;
        if (!loc && warp == 0 && pi + STAGES < packed_tiles) request(pi + STAGES);
        if (!loc && pi + STAGES < packed_tiles) ++issued;
        if (raise) {
            int *const w_max = reinterpret_cast<int *>(p_ptr);           // [4][N]: P is written later
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int m = __reduce_max_sync(0xffffffffu, ordered(x[n]));
                if (lane == 0) w_max[warp * N + n] = m;
            }
            __syncthreads();
            if (tid < N) {
                const float m_old = -neg_m[tid];
                const float mx = unordered(max(max(w_max[tid], w_max[N + tid]), max(w_max[2 * N + tid], w_max[3 * N + tid]))) * p.scale_log2;
                const float m_new = fmaxf(m_old, mx);
                neg_m[tid] = -m_new;
                l_sm[tid] = m_new == -CUDART_INF_F ? 1.f : fast_exp2(m_old - m_new);
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) l[n] *= l_sm[n];
            if (i > 0) {
#pragma unroll
                for (int c = 0; c < N / 16; ++c) {
                    uint32_t v[16];
                    tc_ld16(t_o + lane_base + c * 16, v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * l_sm[c * 16 + e]);
                    tc_st16(t_o + lane_base + c * 16, v);
                }
                tc_wait_st();
            }
        }
#pragma unroll
        for (int c = 0; c < N / 8; ++c) {
            float e[8];
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const float4 m = *reinterpret_cast<const float4 *>(neg_m + 8 * c + k);
                const float mm[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
                for (int u = 0; u < 4; ++u) e[k + u] = fast_exp2(fmaf(x[8 * c + k + u], p.scale_log2, mm[u]));
            }
            if (masked) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (8 * c + k < n_min) e[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) l[8 * c + k] += e[k];
            *reinterpret_cast<uint4 *>(p_ptr + pa_p_chunk<N>(tid, c)) =
                make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7]));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncthreads();
        if (warp == 0) {
            tc_fence_after();
            const uint64_t p_desc = pa_p_desc<N>(base + N * kRowBytes);
#pragma unroll
            for (int k = 0; k < kPaTileCols; ++k)
                tc_mma_bf16_ts(t_o, t_v + 8 * k, p_desc + (uint64_t)((k * 32 * N) >> 4), pa_idesc(N, true), (i > 0 || k) ? 1u : 0u);
            tc_commit(bar_o);
        }
    }
    // ---- epilogue -------------------------------------------------------------------------------------------------
    if (n_tiles > 0 && !*dead && !mbar_wait(bar_o, (n_tiles - 1) & 1, p.err, 84)) *dead = 1;
    if (*dead) {                                                         // nobody leaves while copies are on their way
        if (tid == 0)
            for (int pi = done_tiles; pi < issued; ++pi) mbar_wait(bar_full(pi % STAGES), (pi / STAGES) & 1, p.err, 85);
    }
    tc_fence_after();
    float *const o_sm = reinterpret_cast<float *>(ring);                 // [N][128]
    float *const l_part = reinterpret_cast<float *>(p_ptr);              // [4][N]
    __syncthreads();                                                     // (waits over, P and the ring idle)
    if (n_tiles > 0) {
#pragma unroll
        for (int c = 0; c < N / 16; ++c) {
            uint32_t v[16];
            tc_ld16(t_o + lane_base + c * 16, v);
#pragma unroll
            for (int e = 0; e < 16; ++e) o_sm[(c * 16 + e) * kHeadDim + tid] = __uint_as_float(v[e]);
        }
    }
    // the threads' sums of a row: half of the values change hands in every round, so that lane k ends with rows k, k + 32, ..
#pragma unroll
    for (int w = N / 2, bit = 16; bit >= 1; bit >>= 1) {
        const bool up = lane & bit;
        if (w >= 1) {
#pragma unroll
            for (int k = 0; k < N / 2; ++k)
                if (k < w) {
                    const float give = up ? l[k] : l[k + w], keep = up ? l[k + w] : l[k];
                    l[k] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
                }
            w >>= 1;
        } else {
            l[0] += __shfl_xor_sync(0xffffffffu, l[0], bit);
        }
    }
    // lane's row: bit 16 chose the half of N, bit 8 the quarter, ..
    if (N >= 32) {
#pragma unroll
        for (int k = 0; k < N / 32; ++k) l_part[warp * N + (N / 32) * lane + k] = l[k];
    } else if (!(lane & 1)) {
        l_part[warp * N + (lane >> 1)] = l[0];
    }
    __syncthreads();
    if (tid < N) l_sm[tid] = n_tiles > 0 ? l_part[tid] + l_part[N + tid] + l_part[2 * N + tid] + l_part[3 * N + tid] : 0.f;
    if constexpr (CLUSTER) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
    if (!*dead) {
        // one warp per row; in a cluster, block `split` takes rows split, split + n_splits, ..
        const int first = CLUSTER ? split + p.n_splits * warp : warp, step = CLUSTER ? 4 * p.n_splits : 4, parts = CLUSTER ? p.n_splits : 1;
#pragma unroll 1
        for (int r = first; r < rows; r += step) {
            float m = -CUDART_INF_F, den = 0.f;
            float4 f[CLUSTER ? kPaMaxCluster : 1];
            if constexpr (CLUSTER) {
#pragma unroll
                for (int k = 0; k < kPaMaxCluster; ++k)
                    if (k < parts) f[k] = pa_ld_cluster4(pa_at_rank(o_sm + r * kHeadDim + lane * 4, (uint32_t)k));
                if (lane < parts) {
                    m = -pa_ld_cluster(pa_at_rank(neg_m + r, (uint32_t)lane));
                    den = pa_ld_cluster(pa_at_rank(l_sm + r, (uint32_t)lane));
                }
            } else {
                f[0] = *reinterpret_cast<const float4 *>(o_sm + r * kHeadDim + lane * 4);
                if (lane == 0) {
                    m = -neg_m[r];
                    den = l_sm[r];
                }
            }
            const float top = unordered(__reduce_max_sync(0xffffffffu, ordered(m)));
            float w = m == -CUDART_INF_F ? 0.f : fast_exp2(m - top);
            den *= w;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
            den = __shfl_sync(0xffffffffu, den, 0);
            w *= den > 0.f ? 1.f / den : 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < (CLUSTER ? kPaMaxCluster : 1); ++k) {
                const float wk = __shfl_sync(0xffffffffu, w, k);
                if (k < parts && wk != 0.f) {                            // (a part that saw no key has not written its accumulator)
                    acc.x = fmaf(wk, f[k].x, acc.x);
                    acc.y = fmaf(wk, f[k].y, acc.y);
                    acc.z = fmaf(wk, f[k].z, acc.z);
                    acc.w = fmaf(wk, f[k].w, acc.w);
                }
            }
            const float lse2 = den > 0.f ? top + log2f(den) : den == 0.f ? -CUDART_INF_F : den;
            if (CLUSTER || p.n_splits == 1) {
                const int tq = (row0 + r) / p.G, a = h * p.G + (row0 + r) % p.G;
                const long long o = ((long long)b * p.T + tq) * p.Hq + a;
                reinterpret_cast<uint2 *>(p.out + o * kRowBytes)[lane] = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
                if (p.lse && lane == 0) p.lse[o] = lse2 * kAtLn2;
            } else {
                const long long o = (long long)blockIdx.x * p.group_rows + r;
                reinterpret_cast<float4 *>(p.part_o + o * kHeadDim)[lane] = acc;
                if (lane == 0) p.part_lse[o] = lse2;
            }
        }
    }
    if constexpr (CLUSTER) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");       // nobody leaves while its shared memory is read
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)pa_tmem_cols(N)) : "memory");
}

// Merges the splits of one query row: out = sum_s w_s o_s / sum_s w_s with w_s = 2^(lse_s - max lse).  One warp per row, four output
// dims per thread, the loads of eight splits in flight at a time.
__global__ void __launch_bounds__(256)
packed_combine_kernel(const PackedAttnParams p, int total)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int wi = 8 * blockIdx.x + (threadIdx.x >> 5);
    if (wi >= total) return;
    const int row = wi % p.R, bh = wi / p.R;
    const int b = bh / p.Hkv, h = bh % p.Hkv;
    const int tq = row / p.G, a = h * p.G + row % p.G;
    const int grp = row / p.group_rows, r = row % p.group_rows;
    const long long prow0 = ((long long)bh * p.n_splits * p.n_groups + grp) * p.group_rows + r;     // partial row of split 0
    const long long pstride = (long long)p.n_groups * p.group_rows;
    float mx = -CUDART_INF_F;
    for (int s = lane; s < p.n_splits; s += 32) mx = fmaxf(mx, p.part_lse[prow0 + s * pstride]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float den = 0.f;
    if (mx > -CUDART_INF_F) {
#pragma unroll 1
        for (int s0 = 0; s0 < p.n_splits; s0 += 8) {
            float w[8];
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const bool in = s0 + u < p.n_splits;
                const long long prow = prow0 + (in ? s0 + u : s0) * pstride;
                w[u] = in ? p.part_lse[prow] : -CUDART_INF_F;
                v[u] = reinterpret_cast<const float4 *>(p.part_o + prow * kHeadDim)[lane];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float ws = fast_exp2(w[u] - mx);                   // 0 for the splits past the last one
                acc.x += ws * v[u].x; acc.y += ws * v[u].y; acc.z += ws * v[u].z; acc.w += ws * v[u].w;
                den += ws;
            }
        }
    }
    const bool any = den > 0.f;
    const float inv = any ? 1.f / den : 0.f;
    const long long orow = ((long long)b * p.T + tq) * p.Hq + a;
    reinterpret_cast<uint2 *>(p.out + orow * kRowBytes)[lane] =
        make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (p.lse && lane == 0) p.lse[orow] = any ? (mx + log2f(den)) * kAtLn2 : -CUDART_INF_F;
}

// ---- host side -----------------------------------------------------------------------------------------
struct PackedPlan {
    int n_groups, group_rows, n, n_splits, tiles_per_split;
    bool in_cluster;
    long long items;
    size_t workspace;
};

static PackedPlan packed_plan(const oasis_dims_t *dims, int T, int n_cols, int local_col)
{
    PackedPlan pl;
    const int R = T * (dims->n_q_heads / dims->n_kv_heads);
    pl.n_groups = (R + 63) / 64;
    pl.group_rows = (R + pl.n_groups - 1) / pl.n_groups;
    pl.n = pl.group_rows <= 16 ? 16 : pl.group_rows <= 32 ? 32 : 64;
    const long long items = (long long)dims->batch * dims->n_kv_heads * pl.n_groups;
    const int tiles = (local_col + kPaTileCols - 1) / kPaTileCols + (n_cols > local_col ? 1 : 0);
    // all thread blocks resident at once as far as the tiles can be split
    long long s = items > 0 ? (long long)sm_count() * pa_blocks(pl.n) / items : 1;
    if (s > tiles) s = tiles;
    if (s < 1) s = 1;
    const int most = kPaListCols / kPaTileCols;                          // tiles whose columns a thread block can list
    if ((tiles + s - 1) / s > most) s = (tiles + most - 1) / most;
    pl.in_cluster = s <= kPaMaxCluster;
    pl.tiles_per_split = (int)((tiles + s - 1) / s);
    pl.n_splits = (tiles + pl.tiles_per_split - 1) / pl.tiles_per_split;
    if (pl.n_splits == 1) pl.in_cluster = false;
    pl.items = items * pl.n_splits;
    pl.workspace = pl.n_splits > 1 && !pl.in_cluster ? (size_t)pl.items * pl.group_rows * (kHeadDim + 1) * sizeof(float) : 0;
    return pl;
}

static int check_packed(const oasis_dims_t *dims, int T, int n_cols, int local_col, const char *who)
{
    if (int rc = check_dims(dims)) return rc;
    if (T < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: n_q_tokens %d", who, T);
    if (n_cols < 1 || n_cols > (1 << 26)) return fail(OASIS_ERR_INVALID_ARG, "%s: n_cols %d", who, n_cols);
    if (local_col < 0 || local_col > n_cols || n_cols - local_col > OASIS_MAX_LOCAL_COLS)
        return fail(OASIS_ERR_INVALID_ARG, "%s: local_col %d with %d columns: 0 to %d local columns", who, local_col, n_cols, OASIS_MAX_LOCAL_COLS);
    const int G = dims->n_q_heads / dims->n_kv_heads;
    if ((long long)T * G > 128)
        return fail(OASIS_ERR_UNSUPPORTED, "%s: %lld query rows per KV head > 128", who, (long long)T * G);
    return OASIS_OK;
}

}  // namespace oasis

extern "C" size_t oasis_packed_attn_workspace_bytes(const oasis_dims_t *dims, int32_t n_q_tokens, int32_t n_cols, int32_t local_col)
{
    using namespace oasis;
    if (check_packed(dims, n_q_tokens, n_cols, local_col, "oasis_packed_attn_workspace_bytes") != OASIS_OK) return 0;
    return packed_plan(dims, n_q_tokens, n_cols, local_col).workspace;
}

extern "C" int oasis_packed_attn(const oasis_dims_t *dims, const void *q, int32_t n_q_tokens, const void *packed_pool, const void *hbm_pool,
                                 const int32_t *slot_tbl, const int32_t *blk_tbl, int32_t n_cols, int32_t local_col, const int32_t *seq_len,
                                 float scale, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace oasis;
    const char *who = "oasis_packed_attn";
    if (int rc = check_packed(dims, n_q_tokens, n_cols, local_col, who)) return rc;
    if (!(scale > 0.f) || scale > 3.0e38f) return fail(OASIS_ERR_INVALID_ARG, "%s: scale %g", who, (double)scale);
    if (dims->batch == 0) return OASIS_OK;
    if (!q || !slot_tbl || !blk_tbl || !seq_len || !out || (local_col > 0 && !packed_pool) || (local_col < n_cols && !hbm_pool))
        return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    if (!aligned16(q) || !aligned16(packed_pool) || !aligned16(hbm_pool) || !aligned16(out))
        return fail(OASIS_ERR_INVALID_ARG, "%s: q, packed_pool, hbm_pool and out must be 16-byte aligned", who);
    const PackedPlan pl = packed_plan(dims, n_q_tokens, n_cols, local_col);
    if (pl.workspace > 0) {
        if (!workspace || workspace_bytes < pl.workspace)
            return fail(OASIS_ERR_WORKSPACE, "%s: workspace of %zu bytes required, %zu given", who, pl.workspace,
                        workspace ? workspace_bytes : (size_t)0);
        if (!aligned16(workspace)) return fail(OASIS_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", who);
    }
    const long long total = (long long)dims->batch * dims->n_q_heads * n_q_tokens;
    if (pl.items * pl.group_rows > 0x7fffffffLL || total > 0x7fffffffLL) return fail(OASIS_ERR_UNSUPPORTED, "%s: grid too large", who);

    PackedAttnParams p = {};
    p.q = (const uint8_t *)q; p.packed = (const uint8_t *)packed_pool; p.local = (const uint8_t *)hbm_pool;
    p.slot_tbl = slot_tbl; p.blk_tbl = blk_tbl; p.seq_len = seq_len; p.out = (uint8_t *)out; p.lse = lse; p.err = error_word();
    p.scale_log2 = scale * kAtLog2e;
    p.T = n_q_tokens; p.Hq = dims->n_q_heads; p.Hkv = dims->n_kv_heads; p.G = p.Hq / p.Hkv; p.n_cols = n_cols; p.local_col = local_col;
    p.R = p.T * p.G; p.n_splits = pl.n_splits; p.tiles_per_split = pl.tiles_per_split; p.n_groups = pl.n_groups; p.group_rows = pl.group_rows;
    p.bd = bounds();
    if (pl.workspace > 0) {
        p.part_o = (float *)workspace;
        p.part_lse = p.part_o + (size_t)pl.items * pl.group_rows * kHeadDim;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)pl.n_splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pl.items);
    cfg.blockDim = dim3(kPaThreads);
    cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr;
    cfg.numAttrs = pl.in_cluster ? 2 : 1;
    cudaError_t e;
#define OASIS_PACKED_LAUNCH_AS(N, X)                                                                                          \
    do {                                                                                                                      \
        e = allow_dynamic_shared(reinterpret_cast<const void *>(packed_attn_kernel<N, X>), pa_smem(N));                       \
        if (e == cudaSuccess) prefer_max_shared_carveout(packed_attn_kernel<N, X>);                                           \
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, packed_attn_kernel<N, X>, p);                                      \
    } while (0)
#define OASIS_PACKED_LAUNCH(N)                                                                                                \
    do {                                                                                                                      \
        cfg.dynamicSmemBytes = pa_smem(N);                                                                                    \
        if (pl.in_cluster) OASIS_PACKED_LAUNCH_AS(N, true);                                                                   \
        else OASIS_PACKED_LAUNCH_AS(N, false);                                                                                \
    } while (0)
    if (pl.n == 16) OASIS_PACKED_LAUNCH(16);
    else if (pl.n == 32) OASIS_PACKED_LAUNCH(32);
    else OASIS_PACKED_LAUNCH(64);
#undef OASIS_PACKED_LAUNCH
#undef OASIS_PACKED_LAUNCH_AS
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    if (pl.workspace > 0) {
        cfg.gridDim = dim3((unsigned)((total + 7) / 8));
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        cfg.numAttrs = 1;
        prefer_max_shared_carveout(packed_combine_kernel);
        e = cudaLaunchKernelEx(&cfg, packed_combine_kernel, p, (int)total);
        if (e != cudaSuccess) {
            cudaGetLastError();
            return fail(OASIS_ERR_CUDA, "%s: combine launch: %s", who, cudaGetErrorString(e));
        }
        return check_launch(who);
    }
    return OASIS_OK;
}
