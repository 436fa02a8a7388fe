// Attention over a working set held in 4 bits (packed.cuh), with the local window in bf16.
//
// Work item = (request, KV head, split of the columns), one thread block; all query rows of the KV head, up to 128, share what it
// unpacks.  Two kernels, by the number of rows: packed_attn_kernel (33 to 128) on the 5th-generation tensor cores, and
// packed_attn_few_kernel (up to 32), further down, where every warp works alone.
// packed_attn_kernel: tiles of eight 16-token blocks.  Other than in the bf16 kernels the keys and values, which have to pass through
// registers anyway, are the A operands in tensor memory, and the query rows the columns:
//   S[token][row] = K Q^T    thread = token: 64 B of codes become the token's 128 bf16 dims, 64 columns of its tensor-memory lane
//   O[dim][row]  += V^T P    thread = dim: 8 B of codes per block become the dim's 16 tokens, 8 columns of its lane
// Q (K-major) and P (row-major by token) are the B operands in shared memory.  So 4-bit data crosses shared memory once, bf16 data
// never (as bf16 tiles in shared memory they would be written and read there, 2.5 times the time that HBM takes to bring them).
// A row's logits lie across the threads: the reference maximum that its weights are taken against is shared, comes from the first
// tile, and is raised only when a logit exceeds it by 2^32, which one vote per tile finds out; the rows' sums are kept per thread and
// added up at the end.
// Roles: four warps unpack keys (thread = token), four values (thread = dim), four per 32 rows take the softmax (thread = token),
// one issues the products, one requests entries (bulk copies, one per block, a ring of five or seven tiles).
// Columns that no row sees are left out when the column list of the split is read (compacted in order: the result does not depend
// on the launch).  The local columns, at most one tile, are the first tile of split 0, read straight from global memory while the
// ring fills.  Splits of a row merge inside a thread-block cluster where eight reach, else through the workspace and a second launch.
// Precision: the unpacked keys and values are exact, 2^-20 of what they stand for (the power of two returns in the logits' scale and
// in the output); logits, maxima, sums and accumulators are fp32; both operands of a product have one type, so the weights go to the
// second product in bf16.  Rounded once (half a step, 2^-8 of a weight) they would put an output that one key decides off by up to 2.3
// times as much as its own rounding to bf16 does: the reference lags behind the maximum, so that key's weight is rounded like any other.
// packed_attn_kernel multiplies them as two terms (2^-17; 27.9 -> 30.8 us for 72 rows, ragged; a reference within 2^3 of the maximum,
// whose raises cost more: 34.3).  packed_attn_few_kernel has the second term in the half of a product that up to four rows leave empty:
// 1.00 times the error of the output's own rounding (0.17 % of its norm, against 64 bits), as above 32 rows, where weights rounded once
// had up to 1.65 times as much in a single row (1,500 drawn ones), for 17.0 -> 16.8 us (16 single tokens) and 72.5 -> 73.2 (2 requests x
// 8,194 columns).  From 5 to 32 rows it takes them once, sums them as rounded by a product with ones, and scales its accumulators by the
// ratio of the two sums, so that the error of a key that decides cancels: 1.05 times on average, 1.26 at most over 4,200 drawn cases of
// one KV head.  A second term by products of its own costs there (one term: two) 16 requests x 130 columns, 20 rows 27.4: 30.7 us;
// 2 x 4,098 columns, 8 rows 45.8: 49.1, 16 rows 57.7: 65.0, 20 rows 71.6: 83.5, 32 rows 87.2: 102.1; the bf16 attention rounds its
// weights once too.  Nothing overflows: the local values, which may be of any size, come first, with weights of at most 1 (2^-20 in the
// accumulator's unit); a packed value is at most 2^15, its weight 2^32.
// What bounds it (32 query and 8 KV heads, a graph): up to 8 rows a warp's chain of loads, unpacking, products and softmax at 16 warps per
// SM: no unit is full (issue slots 54 %, integer 43 %, HBM 44 %), and unpacking is 466 of the about 700 instructions that a scheduler
// issues per 128 tokens and 8 rows.  With 1,100 cycles a tile and SM 2 requests x 8,194 columns take 73.2 us (4.1 TB/s; the bf16 kernel
// 171), 16 requests x 130 columns 16.8, 5 of them first loads, list and end (26.4); with 20 rows 27.4, 8 warps per SM, which their
// accumulators allow, and 800 cycles of products a tile (27.2).  From 33 rows on half of a tile's time is its way through
// copies, unpacking, products and softmax and their barriers (3,500 cycles at 72 rows, of which the exponential unit is busy for 768):
// 16 requests x 130 columns 36.4 us under 64 rows, 44.6 under 72, 55.4 under 128; the bf16 kernel, which copies and does not unpack, takes
// 27.5 under 32 rows (here 33.4), 28.1 under 64 and 29.4 under 128, and 94.6 for 2 requests x 4,098 columns under 64 (here 98.4).
#include <cuda.h>
#include <math_constants.h>

#include "packed.cuh"
#include "tc_common.cuh"

namespace oasis {

constexpr int kPaTileCols = 8, kPaTileKeys = kPaTileCols * kBlock;       // 128 tokens: the rows of one MMA
constexpr int kPaStageBytes = kPaTileCols * kPackedBytes;                // 18 KiB
constexpr int kPaMaxCluster = 8;
constexpr float kPaRaise = 32.f;                                         // (log2) how far a logit may exceed its row's reference
// packed_attn_kernel, n = 64, 96 or 128 columns.  Warps: 0-3 keys, 4-7 values, then four per 32 columns for the softmax, one for the
// products, one for the copies.
constexpr int kPaListCols = 2048;                                        // columns of a split at most
__host__ __device__ constexpr int pa_soft(int n) { return 4 * n; }                          // softmax threads
__host__ __device__ constexpr int pa_threads(int n) { return 256 + pa_soft(n) + 64; }
__host__ __device__ constexpr int pa_stages(int n) { return n == 64 ? 7 : 5; }
__host__ __device__ constexpr int pa_k_bufs(int n) { return n == 64 ? 2 : 1; }              // K and V operands in tensor memory
__host__ __device__ constexpr int pa_v_bufs(int n) { return n == 128 ? 1 : 2; }
__host__ __device__ constexpr int pa_tmem_used(int n) { return 64 * (pa_k_bufs(n) + pa_v_bufs(n)) + 3 * n; }     // K | V | two S | O
constexpr int kPaTmemCols = 512;
// Shared memory: Q [dim half][n rows][128 B] | two terms of P [64 columns][128 tokens][128 B] | ring | column list | statistics and barriers.
__host__ __device__ constexpr int pa_p_bytes(int n) { return (n + 63) / 64 * kPaTileKeys * 128; }
__host__ __device__ constexpr int pa_smem(int n)
{
    return 1024 + n * kRowBytes + 2 * pa_p_bytes(n) + pa_stages(n) * kPaStageBytes + kPaListCols * 8 + 2048;
}
static_assert(pa_smem(64) <= 232448 && pa_smem(96) <= 232448 && pa_smem(128) <= 232448, "shared memory of a thread block");
static_assert(pa_tmem_used(64) <= kPaTmemCols && pa_tmem_used(96) <= kPaTmemCols && pa_tmem_used(128) <= kPaTmemCols, "tensor memory");
static_assert(pa_stages(128) * kPaStageBytes >= 128 * kHeadDim * 4, "the accumulator fits into the ring");

struct PackedAttnParams {
    const uint8_t *q, *packed, *local;
    const int32_t *slot_tbl, *blk_tbl, *seq_len;
    uint8_t *out;
    float *lse;
    float *part_o;      // [items][rows][128] fp32, normalised (runs through the workspace only)
    float *part_lse;    // [items][rows]      log2 domain
    int32_t *err;
    float scale_log2;   // of bf16 keys; of unpacked ones: times 2^kDequantShift
    int T, Hq, Hkv, G, n_cols, local_col, R, n_splits, tiles_per_split;
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
// P: rows = tokens of 128 bytes (64 columns), 128-byte swizzle, groups of eight tokens; the next 64 columns 128 rows further.
__device__ __forceinline__ uint32_t pa_p_chunk(int token, int c)         // byte offset of columns 8 c .. 8 c + 7 of a token
{
    return (uint32_t)((c >> 3) * (kPaTileKeys * 128) + token * 128 + (((c ^ token) & 7) << 4));
}

// Named barrier 1 over the softmax threads, returning the OR of their predicates; and the plain barrier 2.
template <int THREADS>
__device__ __forceinline__ bool pa_any(bool pred)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.or.pred q, 1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r) : "r"((uint32_t)pred), "n"(THREADS) : "memory");
    return r != 0;
}
template <int THREADS>
__device__ __forceinline__ void pa_sync()
{
    asm volatile("bar.sync 2, %0;" ::"n"(THREADS) : "memory");
}

// The end of a thread block's work: its rows' accumulators (o_sm, PITCH floats a row, in units of 2^-kDequantShift), reference maxima
// (neg_m, negated, log2) and sums (l_sm) become outputs, or the split's part of them.  `warps` warps take a row each; in a cluster,
// block `split` takes rows split, split + n_splits, .. of all its blocks.  Called by the whole thread block.
template <bool CLUSTER, int PITCH>
__device__ __forceinline__ void pa_finish(const PackedAttnParams &p, bool alive, int warp, int warps, int lane, int split, int rows, int b, int h,
                                          const float *o_sm, const float *neg_m, const float *l_sm)
{
    if constexpr (CLUSTER) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
    if (alive && warp < warps) {
        const int first = CLUSTER ? split + p.n_splits * warp : warp, step = CLUSTER ? warps * p.n_splits : warps, parts = CLUSTER ? p.n_splits : 1;
#pragma unroll 1
        for (int r = first; r < rows; r += step) {
            float m = -CUDART_INF_F, den = 0.f;
            float4 f[CLUSTER ? kPaMaxCluster : 1];
            if constexpr (CLUSTER) {
#pragma unroll
                for (int k = 0; k < kPaMaxCluster; ++k)
                    if (k < parts) f[k] = pa_ld_cluster4(pa_at_rank(o_sm + r * PITCH + lane * 4, (uint32_t)k));
                if (lane < parts) {
                    m = -pa_ld_cluster(pa_at_rank(neg_m + r, (uint32_t)lane));
                    den = pa_ld_cluster(pa_at_rank(l_sm + r, (uint32_t)lane));
                }
            } else {
                f[0] = *reinterpret_cast<const float4 *>(o_sm + r * PITCH + lane * 4);
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
            w *= den == 0.f ? 0.f : 1.f / den;                           // (a query with NaN: NaN)
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
            constexpr float kUnit = (float)(1 << kDequantShift);
            acc.x *= kUnit; acc.y *= kUnit; acc.z *= kUnit; acc.w *= kUnit;
            const float lse2 = den == 0.f ? -CUDART_INF_F : top + log2f(den);
            if (CLUSTER || p.n_splits == 1) {
                const int tq = r / p.G, a = h * p.G + r % p.G;
                const long long o = ((long long)b * p.T + tq) * p.Hq + a;
                reinterpret_cast<uint2 *>(p.out + o * kRowBytes)[lane] = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
                if (p.lse && lane == 0) p.lse[o] = lse2 * kAtLn2;
            } else {
                const long long o = (long long)blockIdx.x * p.R + r;
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
}

// N: columns of the products (query rows, padded).  With 128 (72 registers a thread) 16 to 20 bytes are spilled, with 96 four.
template <int N, bool CLUSTER>
__global__ void __launch_bounds__(pa_threads(N), 1)
packed_attn_kernel(const PackedAttnParams p)
{
    constexpr int STAGES = pa_stages(N), KB = pa_k_bufs(N), VB = pa_v_bufs(N), THREADS = pa_threads(N);
    constexpr int NC = 32;                                  // softmax columns of a thread
    constexpr int SOFT = pa_soft(N);                        // softmax threads
    constexpr int SOFT0 = 8, MMA = SOFT0 + SOFT / 32, COPY = MMA + 1;      // first softmax warp, the others
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    uint8_t *const p_ptr = base_ptr + N * kRowBytes;
    uint8_t *const ring = p_ptr + 2 * pa_p_bytes(N);
    int2 *const list = reinterpret_cast<int2 *>(ring + STAGES * kPaStageBytes);           // (block, slot)
    float *const neg_m = reinterpret_cast<float *>(list + kPaListCols);                     // [N] minus the rows' reference maxima
    float *const l_sm = neg_m + N;                                                          // [N]; while a maximum is raised: factors
    uint64_t *const bars = reinterpret_cast<uint64_t *>(l_sm + N);
    int2 *const s_local = reinterpret_cast<int2 *>(bars + 2 * STAGES + 10);                  // [8] the local columns
    int *const s_cnt = reinterpret_cast<int *>(s_local + kPaTileCols);                      // [columns / 32]
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(s_cnt + kPaListCols / 32);
    const uint32_t bar0 = smem_u32(bars), bar1 = bar0 + 16u * STAGES, bar_p = bar1 + 64u;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (STAGES + s); };
    auto bar_k = [&](int i) { return bar1 + 8u * (i % KB); };           // keys, values of tile i unpacked
    auto bar_v = [&](int i) { return bar1 + 16u + 8u * (i % VB); };
    auto bar_s = [&](int i) { return bar1 + 32u + 8u * (i & 1); };      // logits of tile i there
    auto bar_o = [&](int i) { return bar1 + 48u + 8u * (i & 1); };      // accumulators complete up to tile i
    auto par_k = [&](int i) { return (uint32_t)((i / KB) & 1); };
    auto par_v = [&](int i) { return (uint32_t)((i / VB) & 1); };
    auto par_2 = [&](int i) { return (uint32_t)((i >> 1) & 1); };

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int split = blockIdx.x % p.n_splits, bh = blockIdx.x / p.n_splits;
    const int b = bh / p.Hkv, h = bh % p.Hkv, rows = p.R;
    if (warp == MMA) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)kPaTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 8); }
        for (int k = 0; k < 2; ++k) {
            mbar_init(bar1 + 8u * k, 4);
            mbar_init(bar1 + 16u + 8u * k, 4);
            mbar_init(bar_s(k), 1);
            mbar_init(bar_o(k), 1);
        }
        mbar_init(bar_p, SOFT / 32);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < N) neg_m[tid] = CUDART_INF_F;
    // This launch may have been brought onto the SMs before the previous one ended: what that wrote is read from here on.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- the split's columns ------------------------------------------------------------------------------------
    // Tiles of a row: the local columns (if any), then eight packed columns each.  Thread k < 256 holds the split's columns k, k + 256, ..
    const int has_local = p.n_cols > p.local_col;
    const int t0 = split * p.tiles_per_split, t1 = t0 + p.tiles_per_split;
    const int c0 = max(t0 - has_local, 0) * kPaTileCols, c1 = min((t1 - has_local) * kPaTileCols, p.local_col);
    const int32_t *blk_row = p.blk_tbl + (long long)bh * p.n_cols, *slot_row = p.slot_tbl + (long long)bh * p.n_cols;
    const long long L = p.seq_len[b], last = L + p.T - 1;               // last position that a row sees
    int2 col[kPaListCols / 256];
#pragma unroll
    for (int k = 0; k < kPaListCols / 256; ++k) {
        const int c = c0 + tid + 256 * k;
        col[k] = make_int2(-1, -1);
        if (warp < 8 && c < c1) col[k] = make_int2(blk_row[c], slot_row[c]);
    }
    if (warp == MMA && lane < kPaTileCols && has_local && t0 == 0 && p.local_col + lane < p.n_cols)
        col[0] = make_int2(blk_row[p.local_col + lane], slot_row[p.local_col + lane]);
    // Q: 16 bytes (chunk c of row r) at a time; columns past the rows are zero
#pragma unroll 4
    for (int i = tid; i < N * 16; i += THREADS) {
        const int r = i >> 4, c = i & 15;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const int tq = r / p.G, a = h * p.G + r % p.G;
            v = *reinterpret_cast<const uint4 *>(p.q + (((long long)b * p.T + tq) * p.Hq + a) * kRowBytes + c * 16);
        }
        *reinterpret_cast<uint4 *>(base_ptr + (c >> 3) * (N * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    bool seen[kPaListCols / 256], late = false;
    unsigned got[kPaListCols / 256];
#pragma unroll
    for (int k = 0; k < kPaListCols / 256; ++k) {
        seen[k] = col[k].x >= 0 && (long long)col[k].x * kBlock <= last;
        if (kBoundsCheck && seen[k]) seen[k] = in_range(col[k].y, p.bd.n_slots, p.bd, kErrSlot);
        late |= warp < 8 && seen[k] && (long long)col[k].x * kBlock + kBlock - 1 > L;        // some token of it not every row sees
        got[k] = __ballot_sync(0xffffffffu, seen[k]);
        if (warp < 8 && lane == 0) s_cnt[8 * k + warp] = __popc(got[k]);
    }
    if (warp == MMA && lane < kPaTileCols) s_local[lane] = seen[0] ? col[0] : make_int2(-1, -1);
    tc_fence_before();
    late = __syncthreads_or(late);
    tc_fence_after();
    int count = 0;
#pragma unroll
    for (int k = 0; k < kPaListCols / 256; ++k)
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (w == warp && seen[k]) list[count + __popc(got[k] & ((1u << lane) - 1u))] = col[k];
            count += s_cnt[8 * k + w];
        }
    int do_local = 0;
#pragma unroll
    for (int k = 0; k < kPaTileCols; ++k) do_local |= s_local[k].x >= 0;
    const int packed_tiles = (count + kPaTileCols - 1) / kPaTileCols, n_tiles = do_local + packed_tiles;
    const uint32_t tmem = *tmem_slot, t_s = tmem + 64 * (KB + VB), t_o = t_s + 2 * N;
    auto t_k = [&](int i) { return tmem + 64u * (uint32_t)(i % KB); };
    auto t_v = [&](int i) { return tmem + 64u * (uint32_t)(KB + i % VB); };
    __syncthreads();                                                     // the list is complete

    float *const o_sm = reinterpret_cast<float *>(ring);                 // [N][128], after the last tile
    float *const l_part = reinterpret_cast<float *>(p_ptr);              // [4][N], after the last tile
    bool alive = true;
    if (warp == COPY) {
        // ---------------------------------------------------------------- copies
        int s = 0, pi = 0;
        uint32_t ph = 1;
#pragma unroll 1
        for (; pi < packed_tiles; ++pi) {
            if (pi >= STAGES) alive = mbar_wait_warp(bar_empty(s), ph, p.err, 81);
            if (!alive) break;
            const int n = min(kPaTileCols, count - pi * kPaTileCols);
            if (lane == 0) mbar_arrive_expect_tx(bar_full(s), (uint32_t)(n * kPackedBytes));
            __syncwarp();
            if (lane < n)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(smem_u32(ring) + (uint32_t)(s * kPaStageBytes + lane * kPackedBytes)),
                               "l"(p.packed + (long long)list[pi * kPaTileCols + lane].y * kPackedBytes), "r"((uint32_t)kPackedBytes),
                               "r"(bar_full(s)) : "memory");
            ring_advance(s, ph, 1, STAGES);
        }
        if (!alive)                                                      // nobody leaves while copies are on their way
            for (int k = max(0, pi - STAGES); k < pi; ++k) mbar_wait_warp(bar_full(k % STAGES), (k / STAGES) & 1, p.err, 82);
    } else if (warp == MMA) {
        // ---------------------------------------------------------------- products (the whole warp, converged)
        const uint64_t q_desc = smem_desc_sw128(base), p_desc = smem_desc_sw128_mn(base + N * kRowBytes, kPaTileKeys * 128, 1024);
        auto values = [&](int i) {
            alive = alive && mbar_wait_warp(bar_v(i), par_v(i), p.err, 84) && mbar_wait_warp(bar_p, i & 1, p.err, 85);
            if (!alive) return;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kPaTileCols; ++k)
                tc_mma_bf16_ts(t_o, t_v(i) + 8 * k, p_desc + (uint64_t)((k * 2048) >> 4), pa_idesc(N, true), (i > 0 || k) ? 1u : 0u);
#pragma unroll
            for (int k = 0; k < kPaTileCols; ++k)
                tc_mma_bf16_ts(t_o, t_v(i) + 8 * k, p_desc + (uint64_t)((pa_p_bytes(N) + k * 2048) >> 4), pa_idesc(N, true), 1u);
            tc_commit(bar_o(i));
        };
#pragma unroll 1
        for (int i = 0; i < n_tiles && alive; ++i) {
            alive = mbar_wait_warp(bar_k(i), par_k(i), p.err, 83);
            // (two S buffers: the softmax has read tile i - 2's when its weights came, before V^T P of that tile)
            if (!alive) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < 8; ++k)
                tc_mma_bf16_ts(t_s + (i & 1) * N, t_k(i) + 8 * k, q_desc + (uint64_t)(((k >> 2) * (N * 128) + (k & 3) * 32) >> 4), pa_idesc(N, false),
                               k ? 1u : 0u);
            tc_commit(bar_s(i));
            if (i > 0) values(i - 1);
        }
        if (n_tiles > 0) values(n_tiles - 1);
    } else if (warp < SOFT0) {
        // ---------------------------------------------------------------- unpacking: thread = token (keys) or dim (values)
        const int me = tid & 127, kb = me >> 4, tok = me & 15;
        const bool keys = warp < 4;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        int s = 0;
        uint32_t ph = 0;
#pragma unroll 1
        for (int i = 0; i < n_tiles; ++i) {                              // (a wait that gave up: no more waits)
            const bool loc = do_local && i == 0;
            if (!loc) alive = alive && mbar_wait_warp(bar_full(s), ph, p.err, 87);
            const uint8_t *const stage = ring + s * kPaStageBytes;
            // the product that read this buffer's last tile is over
            if (keys && i >= KB) alive = alive && mbar_wait_warp(bar_s(i - KB), par_2(i - KB), p.err, 88);
            if (!keys && i >= VB) alive = alive && mbar_wait_warp(bar_o(i - VB), par_2(i - VB), p.err, 89);
            tc_fence_after();
            const uint32_t dst = (keys ? t_k(i) : t_v(i)) + lane_base;
            if (loc && keys) {
                const int2 e = s_local[kb];
                const bool any = e.x >= 0 && (long long)e.x * kBlock + tok <= last;         // (others may hold anything)
                const uint4 *src = reinterpret_cast<const uint4 *>(p.local + (long long)(any ? e.y : 0) * kEntryBytes + tok * kRowBytes);
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t r[16];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint4 v = any ? src[4 * c + k] : make_uint4(0, 0, 0, 0);
                        r[4 * k] = v.x; r[4 * k + 1] = v.y; r[4 * k + 2] = v.z; r[4 * k + 3] = v.w;
                    }
                    tc_st16(dst + c * 16, r);
                }
            } else if (loc) {
#pragma unroll 1
                for (int k2 = 0; k2 < kPaTileCols; k2 += 2) {
                    uint32_t r[16];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int2 e = s_local[k2 + u];
                        const uint16_t *src = reinterpret_cast<const uint16_t *>(p.local + (long long)(e.x >= 0 ? e.y : 0) * kEntryBytes + kPartBytes) + me;
                        // tokens past the last visible one may hold anything
                        const int n = e.x >= 0 ? (int)min((long long)kBlock, last - (long long)e.x * kBlock + 1) : 0;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint32_t lo = 2 * j < n ? src[2 * j * kHeadDim] : 0u, hi = 2 * j + 1 < n ? src[(2 * j + 1) * kHeadDim] : 0u;
                            r[8 * u + j] = lo | hi << 16;
                        }
                    }
                    tc_st16(dst + k2 * 8, r);
                }
            } else if (keys) {
                const uint8_t *ent = stage + kb * kPackedBytes;
#pragma unroll 2
                for (int c = 0; c < 4; ++c) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(ent + c * 256 + tok * 16);
                    const uint32_t sc = *reinterpret_cast<const uint16_t *>(ent + kPackedKScale + tok * 8 + c * 2);
                    uint32_t r[16];
                    const DequantScale d0 = dequant_scale(__byte_perm(sc, 0u, 0x4040));
                    const DequantScale d1 = dequant_scale(__byte_perm(sc, 0u, 0x4141));
                    dequant_word(w.x, d0, r);
                    dequant_word(w.y, d0, r + 4);
                    dequant_word(w.z, d1, r + 8);
                    dequant_word(w.w, d1, r + 12);
                    tc_st16(dst + c * 16, r);
                }
            } else {
#pragma unroll 2
                for (int k2 = 0; k2 < kPaTileCols; k2 += 2) {
                    uint32_t r[16];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const uint8_t *ent = stage + (k2 + u) * kPackedBytes;
                        const uint2 w = *reinterpret_cast<const uint2 *>(ent + kPackedV + me * 8);
                        const DequantScale d = dequant_scale(ent[kPackedVScale + me] * 0x00010001u);
                        dequant_word(w.x, d, r + 8 * u);
                        dequant_word(w.y, d, r + 8 * u + 4);
                    }
                    tc_st16(dst + k2 * 8, r);
                }
            }
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(keys ? bar_k(i) : bar_v(i));
                if (!loc) mbar_arrive(bar_empty(s));
            }
            if (!loc) ring_advance(s, ph, 1, STAGES);
        }
    } else {
        // ---------------------------------------------------------------- softmax: thread = token, one logit per query row
        const int me = (tid - 32 * SOFT0) & 127, n0 = (warp - SOFT0) / 4 * NC;        // token of the tile, first column
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const int kb = me >> 4, tok = me & 15;
        uint64_t l2[NC / 2];                                             // sums of the weights, two columns each
#pragma unroll
        for (int n = 0; n < NC / 2; ++n) l2[n] = 0;
#pragma unroll 1
        for (int i = 0; i < n_tiles; ++i) {                              // (a wait that gave up: no more waits, but every barrier)
            const bool loc = do_local && i == 0;
            int n_min = 0;                                               // the first query row that sees this thread's token
            bool masked = false;
            if (late || loc || i == n_tiles - 1) {                       // (elsewhere eight blocks that every row sees whole)
                const int at = (i - do_local) * kPaTileCols + kb;
                const int blk = loc ? s_local[kb].x : at < count ? list[at].x : -1;
                const long long ahead = (long long)blk * kBlock + tok - L;
                n_min = (blk < 0 || ahead >= p.T ? N : ahead <= 0 ? 0 : min((int)ahead * p.G, N)) - n0;
                masked = __any_sync(0xffffffffu, n_min > 0);
            }
            const float scale = loc ? p.scale_log2 : p.scale_log2 * (float)(1 << kDequantShift);
            const uint32_t t_mine = t_s + (i & 1) * N + n0 + lane_base;
            alive = alive && mbar_wait_warp(bar_s(i), par_2(i), p.err, 90);
            tc_fence_after();
            // sixteen columns at a time, as (logit - reference) in log2 units; read a second time for the weights
            float x[16];
            const uint64_t scale2 = f32x2(scale, scale);
            auto read = [&](int c) {
                uint32_t v[16];
                tc_ld16(t_mine + c * 16, v);
#pragma unroll
                for (int n = 0; n < 16; ++n) x[n] = __uint_as_float(v[n]);
                if (masked) {
#pragma unroll
                    for (int n = 0; n < 16; ++n)
                        if (c * 16 + n < n_min) x[n] = -CUDART_INF_F;
                }
            };
            auto relative = [&](int c) {
#pragma unroll
                for (int n = 0; n < 16; n += 4) {
                    const float4 m = *reinterpret_cast<const float4 *>(neg_m + n0 + c * 16 + n);
                    f32x2_split(fma_f32x2(f32x2(x[n], x[n + 1]), scale2, f32x2(m.x, m.y)), x[n], x[n + 1]);
                    f32x2_split(fma_f32x2(f32x2(x[n + 2], x[n + 3]), scale2, f32x2(m.z, m.w)), x[n + 2], x[n + 3]);
                }
            };
            float m4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int c = 0; c < NC / 16; ++c) {
                read(c);
                relative(c);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    m4[n] = max3(m4[n], x[n], x[n + 4]);
                    m4[n] = max3(m4[n], x[n + 8], x[n + 12]);
                }
            }
            const bool raise = pa_any<SOFT>(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) > kPaRaise);
            // V^T P of the tile before has read its weights, and O is complete up to it
            if (i > 0) alive = alive && mbar_wait_warp(bar_o(i - 1), par_2(i - 1), p.err, 86);
            if (raise) {
                // the columns' maxima over the warp's tokens: half of the values change hands in every round
                float *const w_max = reinterpret_cast<float *>(p_ptr);   // [4][N]: P is written later
#pragma unroll 1                                                         // (a rare path: unrolled, it costs the loop registers)
                for (int c = 0; c < NC / 16; ++c) {
                    read(c);
#pragma unroll
                    for (int w = 8; w >= 1; w >>= 1) {
                        const bool up = lane & w;
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k < w) {
                                const float give = up ? x[k] : x[k + w], keep = up ? x[k + w] : x[k];
                                x[k] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, w));
                            }
                    }
                    const float m = fmaxf(x[0], __shfl_xor_sync(0xffffffffu, x[0], 16));
                    if (lane < 16) w_max[(warp & 3) * N + n0 + c * 16 + lane] = m;
                }
                pa_sync<SOFT>();
                const int n = tid - 32 * SOFT0;
                if (n < N) {
                    const float m_old = -neg_m[n];
                    const float mx = fmaxf(fmaxf(w_max[n], w_max[N + n]), fmaxf(w_max[2 * N + n], w_max[3 * N + n])) * scale;
                    const float m_new = fmaxf(m_old, mx);
                    neg_m[n] = -m_new;
                    l_sm[n] = m_new == -CUDART_INF_F ? 1.f : fast_exp2(m_old - m_new);
                }
                pa_sync<SOFT>();
#pragma unroll
                for (int k = 0; k < NC / 2; ++k) l2[k] = fma_f32x2(l2[k], f32x2(l_sm[n0 + 2 * k], l_sm[n0 + 2 * k + 1]), 0);
                if (i > 0) {
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < NC / 16; ++c) {
                        uint32_t v[16];
                        tc_ld16(t_o + n0 + lane_base + c * 16, v);
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * l_sm[n0 + c * 16 + e]);
                        tc_st16(t_o + n0 + lane_base + c * 16, v);
                    }
                    tc_wait_st();
                }
            }
#pragma unroll
            for (int c = 0; c < NC / 16; ++c) {
                read(c);
                relative(c);
#pragma unroll
                for (int n = 0; n < 16; ++n) x[n] = fast_exp2(x[n]);
                if (masked) {
#pragma unroll
                    for (int n = 0; n < 16; ++n)
                        if (c * 16 + n < n_min) x[n] = 0.f;
                }
#pragma unroll
                for (int n = 0; n < 8; ++n) l2[c * 8 + n] = add_f32x2(l2[c * 8 + n], f32x2(x[2 * n], x[2 * n + 1]));
                if (loc) {                                               // the accumulator's unit is 2^-kDequantShift
#pragma unroll
                    for (int n = 0; n < 16; ++n) x[n] *= 1.f / (float)(1 << kDequantShift);
                }
#pragma unroll
                for (int k = 0; k < 16; k += 8) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float a = x[k + 2 * u], c = x[k + 2 * u + 1];
                        hi[u] = pack_bf16x2(a, c);
                        lo[u] = pack_bf16x2(a - __uint_as_float(hi[u] << 16), c - __uint_as_float(hi[u] & 0xffff0000u));
                    }
                    const uint32_t at = pa_p_chunk(me, (n0 + c * 16 + k) / 8);
                    *reinterpret_cast<uint4 *>(p_ptr + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4 *>(p_ptr + pa_p_bytes(N) + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p);
        }
        if (n_tiles > 0) alive = alive && mbar_wait_warp(bar_o(n_tiles - 1), par_2(n_tiles - 1), p.err, 92);
        tc_fence_after();
        // ---- the split's result: accumulators and sums to shared memory (the ring and P are idle)
        if (n_tiles > 0 && alive) {
#pragma unroll
            for (int c = 0; c < NC / 16; ++c) {
                uint32_t v[16];
                tc_ld16(t_o + n0 + lane_base + c * 16, v);
#pragma unroll
                for (int e = 0; e < 16; ++e) o_sm[(n0 + c * 16 + e) * kHeadDim + me] = __uint_as_float(v[e]);
            }
        }
        // the threads' sums of a row: half of the values change hands in every round, so that lane k ends with row k
        float l[NC];
#pragma unroll
        for (int n = 0; n < NC / 2; ++n) f32x2_split(l2[n], l[2 * n], l[2 * n + 1]);
#pragma unroll
        for (int w = NC / 2; w >= 1; w >>= 1) {                          // (lane bit w picks the half)
            const bool up = lane & w;
#pragma unroll
            for (int k = 0; k < NC / 2; ++k)
                if (k < w) {
                    const float give = up ? l[k] : l[k + w], keep = up ? l[k + w] : l[k];
                    l[k] = keep + __shfl_xor_sync(0xffffffffu, give, w);
                }
        }
        l_part[(warp & 3) * N + n0 + lane] = l[0];
    }
    alive = __syncthreads_and(alive);
    if (tid < N) l_sm[tid] = n_tiles > 0 ? l_part[tid] + l_part[N + tid] + l_part[2 * N + tid] + l_part[3 * N + tid] : 0.f;
    pa_finish<CLUSTER, kHeadDim>(p, alive, warp, MMA, lane, split, rows, b, h, o_sm, neg_m, l_sm);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == MMA)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kPaTmemCols) : "memory");
}

// ---- up to 32 query rows: every warp by itself ----------------------------------------------------------------------------
// With few rows the products are small and what a tile costs above is mostly its way through five roles and their barriers: with 16
// columns there, and two thread blocks per SM, 500 of 1,000 instructions of a scheduler per tile and 2,200 cycles of latency, 90.4 us
// for 2 requests x 8,194 columns (16 rows of wider warp products, rows as their 16-row side: 86.5; this: 73.2).  Here a warp takes 32 tokens (two
// blocks) through unpacking, softmax and products alone, with warp-wide products of 16 tokens (or dims) x 8 query rows x 16: no
// barrier but the arrival of its own copies.  The layout of the entries fits the products' operands, because the order of a
// contraction is free.  With lane = (g, t) = (lane / 4, lane % 4):
//   S^T = K Q^T   the lane brings 32 dims, chunk t, of token 8 (t' & 1) + 2 j + e of block t' >> 1, g = 2 t' + e, for j = 0 .. 3
//   O^T += V^T P^T   the lane brings a 32-bit word, tokens 8 (t & 1) .. + 7 of block t >> 1, of dims 16 m + g and + 8
// so that the weights, transposed 8 x 8 (one instruction), are in the order of the words: tokens 2 j and 2 j + 1 of word t.
// Consecutive products go to different accumulators, and with 8 rows the logits have two sets (75.5 -> 71.3 us
// before the weights were summed as rounded).
// NT: products of 8 query rows.  Against it at the change-over, 2 requests x 4,098 columns: 32 rows 87.8 us here, 33 to 64 there 97;
// 40 rows in two thread blocks of 20 here 119, there 83 (both with weights rounded once).  25 to 32 rows spill 36 bytes at 255 registers, 9 to 16
// rows four at 168, 5 to 8 rows in a cluster twelve at 128.
constexpr int kPfThreads = 128, kPfWarps = 4;
constexpr int kPfListCols = 768;                                         // columns of a split at most
constexpr int kPfUnitBytes = 2 * kPackedBytes;
constexpr int kPfPitch = kHeadDim + 4;
__host__ __device__ constexpr int pf_blocks(int nt) { return nt == 1 ? 4 : nt == 2 ? 3 : 2; }       // thread blocks per SM
__host__ __device__ constexpr int pf_stages(int nt) { return nt == 1 ? 2 : nt == 2 ? 3 : 4; }       // units of a warp in flight
// Shared memory: Q fragments | rings | column list | statistics and barriers.
__host__ __device__ constexpr int pf_smem(int nt)
{
    return 128 + nt * 2048 + kPfWarps * pf_stages(nt) * kPfUnitBytes + kPfListCols * 8 + 1536;
}
static_assert((pf_smem(1) + 1024) * pf_blocks(1) <= 233472 && (pf_smem(2) + 1024) * pf_blocks(2) <= 233472 && (pf_smem(3) + 1024) * pf_blocks(3) <= 233472 &&
              (pf_smem(4) + 1024) * pf_blocks(4) <= 233472, "thread blocks per SM");
static_assert(pf_stages(1) * kPfUnitBytes >= 8 * kPfPitch * 4 && pf_stages(2) * kPfUnitBytes >= 16 * kPfPitch * 4 &&
              pf_stages(4) * kPfUnitBytes >= 32 * kPfPitch * 4, "a warp's accumulator fits into its ring");

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// TWO (up to four rows): rows 4 .. 7 of the product repeat rows 0 .. 3, and their weights are what the first four's lose in rounding to
// bf16, so that the weights are two terms for no more products.
template <int NT, bool TWO, bool CLUSTER>
__global__ void __launch_bounds__(kPfThreads, pf_blocks(NT))
packed_attn_few_kernel(const PackedAttnParams p)
{
    static_assert(!TWO || NT == 1, "two terms side by side in one product of eight rows");
    constexpr int STAGES = pf_stages(NT), ROWS = 8 * NT;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const base_ptr = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
    uint4 *const q_frag = reinterpret_cast<uint4 *>(base_ptr);                              // [NT][4 pairs of steps][32 lanes]
    uint8_t *const rings = base_ptr + NT * 2048;
    int2 *const list = reinterpret_cast<int2 *>(rings + kPfWarps * STAGES * kPfUnitBytes);   // (block, slot)
    float *const neg_m = reinterpret_cast<float *>(list + kPfListCols);                       // [warps][ROWS], then [ROWS] of the block
    float *const l_sm = neg_m + kPfWarps * ROWS;
    uint64_t *const bars = reinterpret_cast<uint64_t *>(l_sm + kPfWarps * ROWS);              // [warps][STAGES]
    int2 *const s_local = reinterpret_cast<int2 *>(bars + kPfWarps * STAGES);                 // [8]
    int *const s_cnt = reinterpret_cast<int *>(s_local + kPaTileCols);                        // [columns / 32]

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x % p.n_splits, bh = blockIdx.x / p.n_splits;
    const int b = bh / p.Hkv, h = bh % p.Hkv, rows = p.R;
    const uint32_t bar0 = smem_u32(bars + warp * STAGES);
    uint8_t *const ring = rings + warp * STAGES * kPfUnitBytes;
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar0 + 8u * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // This launch may have been brought onto the SMs before the previous one ended: what that wrote is read from here on.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- the split's columns, as in packed_attn_kernel -----------------------------------------------------------
    constexpr int PER = kPfListCols / kPfThreads;
    const int has_local = p.n_cols > p.local_col;
    const int t0 = split * p.tiles_per_split, t1 = t0 + p.tiles_per_split;
    const int c0 = max(t0 - has_local, 0) * kPaTileCols, c1 = min((t1 - has_local) * kPaTileCols, p.local_col);
    const int32_t *blk_row = p.blk_tbl + (long long)bh * p.n_cols, *slot_row = p.slot_tbl + (long long)bh * p.n_cols;
    const long long L = p.seq_len[b], last = L + p.T - 1;               // last position that a row sees
    int2 col[PER], near = make_int2(-1, -1);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = c0 + tid + kPfThreads * k;
        col[k] = make_int2(-1, -1);
        if (c < c1) col[k] = make_int2(blk_row[c], slot_row[c]);
    }
    if (tid < kPaTileCols && has_local && t0 == 0 && p.local_col + tid < p.n_cols)
        near = make_int2(blk_row[p.local_col + tid], slot_row[p.local_col + tid]);
    // Q as the lanes of a product hold it: pair k of steps, lane (g, t): dims 32 t + 8 k .. + 7 of row g
    for (int i = tid; i < NT * 128; i += kPfThreads) {
        const int lt = i & 31, k = (i >> 5) & 3, row = TWO ? (lt >> 2) & 3 : (i >> 7) * 8 + (lt >> 2);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < rows) {
            const int tq = row / p.G, a = h * p.G + row % p.G;
            v = *reinterpret_cast<const uint4 *>(p.q + (((long long)b * p.T + tq) * p.Hq + a) * kRowBytes + (32 * (lt & 3) + 8 * k) * 2);
        }
        q_frag[i] = v;
    }
    bool seen[PER], late = false;
    unsigned got[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        seen[k] = col[k].x >= 0 && (long long)col[k].x * kBlock <= last;
        if (kBoundsCheck && seen[k]) seen[k] = in_range(col[k].y, p.bd.n_slots, p.bd, kErrSlot);
        late |= seen[k] && (long long)col[k].x * kBlock + kBlock - 1 > L;                    // some token of it not every row sees
        got[k] = __ballot_sync(0xffffffffu, seen[k]);
        if (lane == 0) s_cnt[4 * k + warp] = __popc(got[k]);
    }
    if (warp == 0) {
        bool ok = near.x >= 0 && (long long)near.x * kBlock <= last;
        if (kBoundsCheck && ok) ok = in_range(near.y, p.bd.n_slots, p.bd, kErrSlot);
        if (lane < kPaTileCols) s_local[lane] = ok ? near : make_int2(-1, -1);
    }
    late = __syncthreads_or(late);
    int count = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int w = 0; w < kPfWarps; ++w) {
            if (w == warp && seen[k]) list[count + __popc(got[k] & ((1u << lane) - 1u))] = col[k];
            count += s_cnt[4 * k + w];
        }
    __syncthreads();                                                     // the list is complete

    // Lanes 0 and 1: the entries of the warp's unit k (units warp, warp + 4, ..) into its stage.
    const int n_units = (count + 1) / 2, mine = n_units > warp ? (n_units - warp + kPfWarps - 1) / kPfWarps : 0;
    auto request = [&](int k, int s) {
        const int at = 2 * (warp + kPfWarps * k), n = min(2, count - at);
        if (lane == 0) mbar_arrive_expect_tx(bar0 + 8u * s, (uint32_t)(n * kPackedBytes));
        __syncwarp();
        if (lane < n)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_u32(ring) + (uint32_t)(s * kPfUnitBytes + lane * kPackedBytes)),
                           "l"(p.packed + (long long)list[at + lane].y * kPackedBytes), "r"((uint32_t)kPackedBytes), "r"(bar0 + 8u * s) : "memory");
    };
#pragma unroll 1
    for (int k = 0; k < min(STAGES, mine); ++k) request(k, k);

    float o[NT][8][4], m_neg[NT][2], l[NT][2];                           // accumulators: dims 16 m + g, + 8; rows 8 nt + 2 t, + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int m = 0; m < 8; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][m][e] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) { m_neg[nt][e] = CUDART_INF_F; l[nt][e] = 0.f; }
    }
    float lw[NT][4];                                                     // sums of the rounded weights (elements 0 and 1)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) lw[nt][0] = lw[nt][1] = lw[nt][2] = lw[nt][3] = 0.f;
    float s[NT][4][2];                                                   // logits of a unit: token j of this lane, rows 2 t and 2 t + 1
    uint32_t pw[NT][4];                                                  // weights of a unit, as the operand of V^T P^T
    const int row0 = TWO ? 2 * (t & 1) : 2 * t;                          // this lane's query rows 8 nt + row0, + 1
    const float less = TWO && t >= 2 ? 1.f : 0.f;                        // the weights' second term
    const int kblk = g >> 2, ktok = 8 * ((g >> 1) & 1) + (g & 1);        // keys: token ktok + 2 j of block kblk
    // From logits to weights.  blk: the block of this lane's tokens; `mask`: some token may be hidden.
    auto softmax = [&](int blk, bool mask, float scale, float unit) {
        if (mask) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const long long ahead = (long long)blk * kBlock + ktok + 2 * j - L;
                const int n_min = blk < 0 || ahead >= p.T ? ROWS : ahead <= 0 ? 0 : min((int)ahead * p.G, ROWS);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (8 * nt + row0 + e < n_min) s[nt][j][e] = -CUDART_INF_F;
            }
        }
        float top = -CUDART_INF_F;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                top = max3(top, fmaf(s[nt][j][0], scale, m_neg[nt][0]), fmaf(s[nt][j][1], scale, m_neg[nt][1]));
        if (__any_sync(0xffffffffu, top > kPaRaise)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = fmaxf(fmaxf(s[nt][0][e], s[nt][1][e]), fmaxf(s[nt][2][e], s[nt][3][e]));
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                    const float m_new = fmaxf(-m_neg[nt][e], mx * scale);
                    const float f = m_new == -CUDART_INF_F ? 1.f : fast_exp2(-m_neg[nt][e] - m_new);
                    m_neg[nt][e] = -m_new;
                    l[nt][e] *= f;
                    lw[nt][e] *= f;
#pragma unroll
                    for (int m = 0; m < 8; ++m) { o[nt][m][e] *= f; o[nt][m][2 + e] *= f; }
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float a = fast_exp2(fmaf(s[nt][j][0], scale, m_neg[nt][0])), c = fast_exp2(fmaf(s[nt][j][1], scale, m_neg[nt][1]));
                if (mask) {
                    if (s[nt][j][0] == -CUDART_INF_F) a = 0.f;
                    if (s[nt][j][1] == -CUDART_INF_F) c = 0.f;
                }
                l[nt][0] += a;
                l[nt][1] += c;
                a *= unit;
                c *= unit;
                uint32_t w = pack_bf16x2(a, c);
                if (TWO) w = pack_bf16x2(fmaf(-less, __uint_as_float(w << 16), a), fmaf(-less, __uint_as_float(w & 0xffff0000u), c));
                pw[nt][j] = transpose_8x8(w);
            }
    };
    // One more row of V^T, of ones: the sums of the weights as the product takes them.
    auto count_weights = [&](uint32_t one) {
        if (TWO) return;                                                 // (two terms: nothing to make good)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mma_16x8x16(lw[nt], one, one, one, one, pw[nt][0], pw[nt][1]);
            mma_16x8x16(lw[nt], one, one, one, one, pw[nt][2], pw[nt][3]);
        }
    };
    // S^T of four tokens per lane: tokens 0, 1 are rows g, g + 8 of the first product, 2, 3 of the second.
    constexpr int KS = NT == 1 ? 2 : 1;                                  // two accumulators where there are few products: shorter chains
    float acc[KS][NT][2][4];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][nt][0][e] = acc[i][nt][1][e] = 0.f;
    };
    auto logits = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s[nt][j][e] = acc[0][nt][j >> 1][2 * (j & 1) + e];
#pragma unroll
                    for (int i = 1; i < KS; ++i) s[nt][j][e] += acc[i][nt][j >> 1][2 * (j & 1) + e];
                }
    };

    // ---- the local columns: unit k of two blocks is warp 3 - k's, straight from global memory
    const int2 la = s_local[2 * (3 - warp)], lb = s_local[2 * (3 - warp) + 1];
    if (la.x >= 0 || lb.x >= 0) {
        clear();
        const int2 kl = kblk ? lb : la, vl = t >> 1 ? lb : la;
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {                                    // dims 32 t + 8 k .. + 7
            uint4 w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int tok = ktok + 2 * j;
                w[j] = make_uint4(0, 0, 0, 0);
                if (kl.x >= 0 && (long long)kl.x * kBlock + tok <= last)                    // (others may hold anything)
                    w[j] = *reinterpret_cast<const uint4 *>(p.local + (long long)kl.y * kEntryBytes + tok * kRowBytes + (32 * t + 8 * k) * 2);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint4 q = q_frag[(nt * 4 + k) * 32 + lane];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    mma_16x8x16(acc[0][nt][m], w[2 * m].x, w[2 * m + 1].x, w[2 * m].y, w[2 * m + 1].y, q.x, q.y);
                    mma_16x8x16(acc[0][nt][m], w[2 * m].z, w[2 * m + 1].z, w[2 * m].w, w[2 * m + 1].w, q.z, q.w);
                }
            }
        }
        logits();
        softmax(kl.x, true, p.scale_log2, 1.f / (float)(1 << kDequantShift));
        count_weights(0x00010001u * ((127u + kDequantShift) << 7));
        const uint16_t *src = reinterpret_cast<const uint16_t *>(p.local + (long long)(vl.x >= 0 ? vl.y : 0) * kEntryBytes + kPartBytes) + 8 * (t & 1) * kHeadDim + g;
        const int n = vl.x >= 0 ? (int)min(8ll, max(0ll, last - ((long long)vl.x * kBlock + 8 * (t & 1)) + 1)) : 0;
#pragma unroll
        for (int m = 0; m < 8; ++m) {                                    // dims 16 m + g, + 8
            uint32_t w[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t lo = 2 * k < n ? src[2 * k * kHeadDim + 16 * m + 8 * u] : 0u, hi = 2 * k + 1 < n ? src[(2 * k + 1) * kHeadDim + 16 * m + 8 * u] : 0u;
                    w[u][k] = lo | hi << 16;
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                mma_16x8x16(o[nt][m], w[0][0], w[1][0], w[0][1], w[1][1], pw[nt][0], pw[nt][1]);
                mma_16x8x16(o[nt][m], w[0][2], w[1][2], w[0][3], w[1][3], pw[nt][2], pw[nt][3]);
            }
        }
    }

    // ---- the packed columns
    bool alive = true;
    int st = 0, k = 0;
    uint32_t ph = 0;
    const float scale = p.scale_log2 * (float)(1 << kDequantShift);
#pragma unroll 1
    for (; k < mine; ++k) {
        alive = __all_sync(0xffffffffu, mbar_wait(bar0 + 8u * st, ph, p.err, 93));
        if (!alive) break;
        const uint8_t *const stage = ring + st * kPfUnitBytes;
        clear();
        {
            const uint8_t *const ent = stage + kblk * kPackedBytes;
            uint4 w[4];
            uint32_t sc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = *reinterpret_cast<const uint4 *>(ent + 256 * t + 16 * (ktok + 2 * j));
                sc[j] = *reinterpret_cast<const uint16_t *>(ent + kPackedKScale + 8 * (ktok + 2 * j) + 2 * t);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                DequantScale d[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) d[j] = dequant_scale(__byte_perm(sc[j], 0u, half ? 0x4141 : 0x4040));
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t v[4][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) dequant_word(half ? (u ? w[j].w : w[j].z) : (u ? w[j].y : w[j].x), d[j], v[j]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint4 q = q_frag[(nt * 4 + half * 2 + u) * 32 + lane];
#pragma unroll
                        for (int m = 0; m < 2; ++m) mma_16x8x16(acc[(2 * u) % KS][nt][m], v[2 * m][0], v[2 * m + 1][0], v[2 * m][1], v[2 * m + 1][1], q.x, q.y);
#pragma unroll
                        for (int m = 0; m < 2; ++m) mma_16x8x16(acc[(2 * u + 1) % KS][nt][m], v[2 * m][2], v[2 * m + 1][2], v[2 * m][3], v[2 * m + 1][3], q.z, q.w);
                    }
                }
            }
        }
        const int at = 2 * (warp + kPfWarps * k) + kblk;
        const bool mask = late || 2 * (warp + kPfWarps * k) + 2 > count;
        logits();
        softmax(mask ? (at < count ? list[at].x : -1) : 0, mask, scale, 1.f);
        count_weights(0x3f803f80u);
        {
            const uint8_t *const ent = stage + (t >> 1) * kPackedBytes;
#pragma unroll
            for (int m2 = 0; m2 < 8; m2 += 2) {                          // dims 16 m + g, + 8
                uint32_t v[2][2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int dim = 16 * (m2 + i) + 8 * u + g;
                        const uint32_t w = *reinterpret_cast<const uint32_t *>(ent + kPackedV + 8 * dim + 4 * (t & 1));
                        dequant_word(w, dequant_scale(ent[kPackedVScale + dim] * 0x00010001u), v[i][u]);
                    }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) mma_16x8x16(o[nt][m2 + i], v[i][0][0], v[i][1][0], v[i][0][1], v[i][1][1], pw[nt][0], pw[nt][1]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) mma_16x8x16(o[nt][m2 + i], v[i][0][2], v[i][1][2], v[i][0][3], v[i][1][3], pw[nt][2], pw[nt][3]);
                }
            }
        }
        __syncwarp();                                                    // the stage has been read
        if (k + STAGES < mine) request(k + STAGES, st);
        ring_advance(st, ph, 1, STAGES);
    }
    if (!alive)                                                          // nobody leaves while copies are on their way
        for (int j = 1; j < STAGES && k + j < mine; ++j) mbar_wait(bar0 + 8u * ((k + j) % STAGES), ((k + j) / STAGES) & 1, p.err, 94);
    // ---- the warps' results come together
    float *const o_mine = reinterpret_cast<float *>(ring);               // [ROWS][kPfPitch]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[nt][e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            const int r = 8 * nt + 2 * t + e;
            const float fit = TWO || lw[nt][e] == 0.f ? 1.f : __fdividef(sum, lw[nt][e]);  // (the accumulators are of rounded weights)
            if (g == 0) {
                neg_m[warp * ROWS + r] = m_neg[nt][e];
                l_sm[warp * ROWS + r] = sum;
            }
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                float lo = o[nt][m][e], hi = o[nt][m][2 + e];
                if (TWO) {                                               // both terms, in either row
                    lo += __shfl_xor_sync(0xffffffffu, lo, 2);
                    hi += __shfl_xor_sync(0xffffffffu, hi, 2);
                }
                o_mine[r * kPfPitch + 16 * m + g] = lo * fit;
                o_mine[r * kPfPitch + 16 * m + g + 8] = hi * fit;
            }
        }
    }
    alive = __syncthreads_and(alive);
    float *const o_sm = reinterpret_cast<float *>(rings);
    constexpr int kPart = STAGES * kPfUnitBytes / 4;                     // floats between the warps' accumulators
#pragma unroll 1
    for (int r = warp; r < rows; r += kPfWarps) {
        float m[kPfWarps], top = -CUDART_INF_F, den = 0.f;
#pragma unroll
        for (int w = 0; w < kPfWarps; ++w) {
            m[w] = -neg_m[w * ROWS + r];
            top = fmaxf(top, m[w]);
        }
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kPfWarps; ++w) {
            const float f = m[w] == -CUDART_INF_F ? 0.f : fast_exp2(m[w] - top);
            const float4 v = *reinterpret_cast<const float4 *>(o_sm + w * kPart + r * kPfPitch + lane * 4);
            den = fmaf(f, l_sm[w * ROWS + r], den);
            acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
        }
        *reinterpret_cast<float4 *>(o_sm + r * kPfPitch + lane * 4) = acc;
        __syncwarp();
        if (lane == 0) {                                                 // (the row's places of warp 0, which only this warp reads)
            neg_m[r] = -top;
            l_sm[r] = den;
        }
    }
    pa_finish<CLUSTER, kPfPitch>(p, alive, warp, kPfWarps, lane, split, rows, b, h, o_sm, neg_m, l_sm);
}

// Merges the splits of one query row: out = sum_s w_s o_s / sum_s w_s with w_s = 2^(lse_s - max lse).  One warp per row, four output
// dims per thread, the loads of eight splits in flight at a time.
__global__ void __launch_bounds__(256)
packed_combine_kernel(const PackedAttnParams p, int total)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // (behind the wait: the splits' launch is over for the next one too)
    const int lane = threadIdx.x & 31;
    const int wi = 8 * blockIdx.x + (threadIdx.x >> 5);
    if (wi >= total) return;
    const int row = wi % p.R, bh = wi / p.R;
    const int b = bh / p.Hkv, h = bh % p.Hkv;
    const int tq = row / p.G, a = h * p.G + row % p.G;
    const long long prow0 = (long long)bh * p.n_splits * p.R + row, pstride = p.R;      // partial row of split 0, from split to split
    float mx = -CUDART_INF_F;
    bool nan = false;
    for (int s = lane; s < p.n_splits; s += 32) {
        const float v = p.part_lse[prow0 + s * pstride];
        mx = fmaxf(mx, v);
        nan |= v != v;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float den = 0.f;
    if (__any_sync(0xffffffffu, nan)) mx = CUDART_NAN_F;
    if (mx != -CUDART_INF_F) {
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
    const bool any = den != 0.f;
    const float inv = any ? 1.f / den : 0.f;
    const long long orow = ((long long)b * p.T + tq) * p.Hq + a;
    reinterpret_cast<uint2 *>(p.out + orow * kRowBytes)[lane] =
        make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (p.lse && lane == 0) p.lse[orow] = any ? (mx + log2f(den)) * kAtLn2 : -CUDART_INF_F;
}

// ---- host side -----------------------------------------------------------------------------------------
struct PackedPlan {
    int rows, n, n_splits, tiles_per_split;         // query rows per KV head; columns of the products
    bool in_cluster;
    long long items;
    size_t workspace;
};

static PackedPlan packed_plan(const oasis_dims_t *dims, int T, int n_cols, int local_col)
{
    PackedPlan pl;
    const int R = T * (dims->n_q_heads / dims->n_kv_heads);
    pl.rows = R;
    pl.n = R <= 32 ? (R + 7) / 8 * 8 : R <= 64 ? 64 : R <= 96 ? 96 : 128;
    const bool few = pl.n <= 32;
    const long long items = (long long)dims->batch * dims->n_kv_heads;
    const int tiles = (local_col + kPaTileCols - 1) / kPaTileCols + (n_cols > local_col ? 1 : 0);
    const int most = (few ? kPfListCols : kPaListCols) / kPaTileCols;    // tiles whose columns a thread block can list
    const int least = (tiles + most - 1) / most, blocks = few ? pf_blocks(pl.n / 8) : 1, sms = sm_count();
    // The number of splits with the smallest estimate, in the time that a thread block alone on an SM takes for a tile: 3 for its
    // first loads and its end, then its tiles, slower by 0.7 for every thread block beyond the first that shares the SM; a wave of them
    // after the other; 0.5 for a merge in a cluster, 2.5 through the workspace.  Candidates: what a cluster holds, and what fills the
    // SMs with one, two, .. thread blocks.  Measured against it, in a graph, one token, 32 query and 8 KV heads (splits: us):
    //   16 requests x 130 columns  1: 20.2  2: 17.2  3: 19.0  4: 17.5  6: 23.0      40 requests  1: 39.4  2: 38.7  3: 35.7  4: 43.3
    //   1 request x 130 columns  1: 18.3  4: 9.0  6: 7.4  8: 7.4  9: 9.2            2 x 4,098 columns  8: 83.2  18: 46.1  27: 43.4  37: 44.6
    //   16 requests x 130 columns, 4 tokens (three thread blocks per SM)  1: 26.8  2: 27.1  3: 22.0  4: 34.1
    //   5 tokens (two)  1: 31.9  2: 27.4  3: 39.5     72 rows (one)  1: 44.6  2: 65.6
    const float share = few ? 0.7f : 1.f;
    long long best = 0;
    float best_cost = 0.f;
    auto consider = [&](long long s) {
        s = s > tiles ? tiles : s;
        s = s < least ? least : s;
        s = s < 1 ? 1 : s;
        const long long per = (tiles + s - 1) / s;
        if (per > 0) s = (tiles + per - 1) / per;                        // (no split without a tile)
        const long long on_sm = (items * s + sms - 1) / sms, waves = (on_sm + blocks - 1) / blocks;
        long long rest = on_sm - (waves - 1) * blocks;
        if (blocks == 3 && on_sm > 1 && rest < blocks && s % 2 == 0) ++rest;     // (three places per SM: pairs of a cluster fill them unevenly)
        auto wave = [&](long long n) { return 3.f + (float)per * (share * (float)n > 1.f ? share * (float)n : 1.f); };
        const float cost = (float)(waves - 1) * wave(blocks) + wave(rest) + (s == 1 ? 0.f : s <= kPaMaxCluster ? 0.5f : 2.5f);
        if (best == 0 || cost < best_cost) {
            best = s;
            best_cost = cost;
        }
    };
    if (items > 0) {
        for (int s = 1; s <= kPaMaxCluster; ++s)
            if (few || s == 1 || clusters_at_once(s) >= items) consider(s);      // (one thread block per SM: all clusters at once)
        for (int k = 1; k <= blocks; ++k) consider((long long)sms * k / items);
    }
    const long long s = best > 0 ? best : 1;
    pl.tiles_per_split = (int)((tiles + s - 1) / s);
    pl.n_splits = pl.tiles_per_split > 0 ? (tiles + pl.tiles_per_split - 1) / pl.tiles_per_split : 1;
    pl.in_cluster = pl.n_splits > 1 && pl.n_splits <= kPaMaxCluster && (few || clusters_at_once(pl.n_splits) >= items);
    pl.items = items * pl.n_splits;
    pl.workspace = pl.n_splits > 1 && !pl.in_cluster ? (size_t)pl.items * pl.rows * (kHeadDim + 1) * sizeof(float) : 0;
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
    if (!(scale > 0.f) || scale > 1.0e30f) return fail(OASIS_ERR_INVALID_ARG, "%s: scale %g", who, (double)scale);
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
    if (pl.items * pl.rows > 0x7fffffffLL || total > 0x7fffffffLL) return fail(OASIS_ERR_UNSUPPORTED, "%s: grid too large", who);

    PackedAttnParams p = {};
    p.q = (const uint8_t *)q; p.packed = (const uint8_t *)packed_pool; p.local = (const uint8_t *)hbm_pool;
    p.slot_tbl = slot_tbl; p.blk_tbl = blk_tbl; p.seq_len = seq_len; p.out = (uint8_t *)out; p.lse = lse; p.err = error_word();
    p.scale_log2 = scale * kAtLog2e;
    p.T = n_q_tokens; p.Hq = dims->n_q_heads; p.Hkv = dims->n_kv_heads; p.G = p.Hq / p.Hkv; p.n_cols = n_cols; p.local_col = local_col;
    p.R = p.T * p.G; p.n_splits = pl.n_splits; p.tiles_per_split = pl.tiles_per_split;
    p.bd = bounds();
    if (pl.workspace > 0) {
        p.part_o = (float *)workspace;
        p.part_lse = p.part_o + (size_t)pl.items * pl.rows * kHeadDim;
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
    cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr;
    cfg.numAttrs = pl.in_cluster ? 2 : 1;
    cudaError_t e;
#define OASIS_PACKED_LAUNCH_AS(...)                                                                                           \
    do {                                                                                                                      \
        e = allow_dynamic_shared(reinterpret_cast<const void *>(__VA_ARGS__), (int)cfg.dynamicSmemBytes);                     \
        if (e == cudaSuccess) prefer_max_shared_carveout(__VA_ARGS__);                                                        \
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, __VA_ARGS__, p);                                                   \
    } while (0)
#define OASIS_PACKED_LAUNCH(THREADS, SMEM, KERNEL, ...)                                                                       \
    do {                                                                                                                      \
        cfg.blockDim = dim3(THREADS);                                                                                         \
        cfg.dynamicSmemBytes = SMEM;                                                                                          \
        if (pl.in_cluster) OASIS_PACKED_LAUNCH_AS(KERNEL<__VA_ARGS__, true>);                                                 \
        else OASIS_PACKED_LAUNCH_AS(KERNEL<__VA_ARGS__, false>);                                                              \
    } while (0)
    if (pl.rows <= 4) OASIS_PACKED_LAUNCH(kPfThreads, pf_smem(1), packed_attn_few_kernel, 1, true);
    else if (pl.n == 8) OASIS_PACKED_LAUNCH(kPfThreads, pf_smem(1), packed_attn_few_kernel, 1, false);
    else if (pl.n == 16) OASIS_PACKED_LAUNCH(kPfThreads, pf_smem(2), packed_attn_few_kernel, 2, false);
    else if (pl.n == 24) OASIS_PACKED_LAUNCH(kPfThreads, pf_smem(3), packed_attn_few_kernel, 3, false);
    else if (pl.n == 32) OASIS_PACKED_LAUNCH(kPfThreads, pf_smem(4), packed_attn_few_kernel, 4, false);
    else if (pl.n == 64) OASIS_PACKED_LAUNCH(pa_threads(64), pa_smem(64), packed_attn_kernel, 64);
    else if (pl.n == 96) OASIS_PACKED_LAUNCH(pa_threads(96), pa_smem(96), packed_attn_kernel, 96);
    else OASIS_PACKED_LAUNCH(pa_threads(128), pa_smem(128), packed_attn_kernel, 128);
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
