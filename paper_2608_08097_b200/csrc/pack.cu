// Blocks of the KV cache in 4 bits: packing (from entries of a pool, from the local window, from a dense pool's separate key and
// value blocks) and unpacking.  The format and its arithmetic are in packed.cuh.
//
// Packing: two warps per (request, block, KV head), one for the keys and one for the values.  Eight 16-byte loads per lane bring the
// 4 KiB: a lane holds the same eight dims of eight tokens, 0 .. 7 in lanes 0 .. 15 and 8 .. 15 in lanes 16 .. 31, so that its eight
// codes of a key are one word, and so are its eight codes of a dim's values.  The largest magnitude of a key's group (16 dims of a
// token) is one exchange with the neighbouring lane away, of a value's group (16 tokens of a dim) seven maxima and one exchange
// with the other half-warp.  Divisions are table look-ups by shuffle, a value is rounded by one fused multiply-add, and four codes
// come together in three integer ones (packed.cuh).  What does not fit into the scales (NaN, infinity, magnitudes above 26,880) is
// found in the groups' maxima and replaced before.  The part is put together in shared memory and leaves in 16-byte stores, whole
// lines, because its place is usually in pinned host memory.  The block's summaries (minimum and maximum of the keys) come from
// the same registers.  Algorithmic traffic: 8,192 B read, 2,304 B (and 512 B of summaries) written per (block, head).
// Measured in device memory, 16,384 entries (a request of 32 K tokens, 8 heads): packing 39.3 us, 4.6 TB/s.  No unit is full there
// (issue slots 52 %, integer 47 %, HBM 43 %): a warp loads once, computes once and stores once, and 24 warps per SM (80 registers) do
// not cover it.  The hand-over of 131,072 dense entries (1 GiB): 280 us into device memory, 5.73 ms into pinned host memory, where the
// link bounds it (52.7 GB/s).  Unpacking 28.6 us, 6.0 TB/s, near what a copy reaches.
// (Both with one warp per entry, divisions and two roundings: 115 us.)  One block of one head: 4.0 us, two dependent launches.
#include "packed.cuh"

namespace oasis {

constexpr int kPackWarps = 4;                               // of a thread block: two entries (unpacking: four)

__device__ __forceinline__ uint32_t bf2_min(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf2_max(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
// NaN counts as zero, what is above the largest value that a scale reaches as that.
__device__ __forceinline__ uint32_t packable(uint32_t v)
{
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t x = (v >> (16 * e)) & 0xffffu, mag = x & 0x7fffu;
        r |= (mag > 0x7f80u ? 0u : mag > kPackLargest ? (x & 0x8000u) | kPackLargest : x) << (16 * e);
    }
    return r;
}
// Maximum of two pairs of magnitudes (bf16 patterns without sign; NaN is the largest).
__device__ __forceinline__ uint32_t bf2_max_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// The keys (KEYS) or the values of one block and head, lane -> 16-byte chunk (lane & 15) of token 8 (lane >> 4) + i, into their part
// of an entry: `steps` and `inverses` are this lane's of the tables, `sm` holds 1,152 bytes of this warp (codes, then scales),
// 16-byte aligned; `dst`: the packed entry.
template <bool KEYS>
__device__ __forceinline__ void pack_part(uint32_t (&x)[8][4], uint32_t steps, float inverses, uint8_t *sm, uint8_t *dst)
{
    const int lane = threadIdx.x & 31, upper = lane >> 4, chunk = lane & 15;
    uint32_t most[8];                                                // the groups' largest magnitudes: of token i, or of dim 8 chunk + i
    auto maxima = [&]() {
        uint32_t all = 0;
        if (KEYS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t a2 = bf2_max_nan(bf2_max_nan(x[i][0] & 0x7fff7fffu, x[i][1] & 0x7fff7fffu), bf2_max_nan(x[i][2] & 0x7fff7fffu, x[i][3] & 0x7fff7fffu));
                a2 = bf2_max_nan(a2, __shfl_xor_sync(0xffffffffu, a2, 1));
                most[i] = max(a2 & 0xffffu, a2 >> 16);
                all = max(all, most[i]);
            }
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                uint32_t a2 = x[0][p] & 0x7fff7fffu;
#pragma unroll
                for (int i = 1; i < 8; ++i) a2 = bf2_max_nan(a2, x[i][p] & 0x7fff7fffu);
                a2 = bf2_max_nan(a2, __shfl_xor_sync(0xffffffffu, a2, 16));
                most[2 * p] = a2 & 0xffffu;
                most[2 * p + 1] = a2 >> 16;
                all = max(all, max(most[2 * p], most[2 * p + 1]));
            }
        }
        return all;
    };
    if (__any_sync(0xffffffffu, maxima() > kPackLargest)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int p = 0; p < 4; ++p) x[i][p] = packable(x[i][p]);
        maxima();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int byte = scale_byte(most[i], steps);
        const float inv = scale_inverse(byte, inverses);
        uint32_t c[8];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (KEYS) {                                              // dims of token 8 upper + i
                c[2 * p] = code_bits(bf_lo(x[i][p]), inv);
                c[2 * p + 1] = code_bits(bf_hi(x[i][p]), inv);
            } else {                                                 // tokens of dim 8 chunk + i
                c[2 * p] = code_bits(i & 1 ? bf_hi(x[2 * p][i >> 1]) : bf_lo(x[2 * p][i >> 1]), inv);
                c[2 * p + 1] = code_bits(i & 1 ? bf_hi(x[2 * p + 1][i >> 1]) : bf_lo(x[2 * p + 1][i >> 1]), inv);
            }
        }
        const uint32_t word = __byte_perm(code_half(c[0], c[2], c[4], c[6]), code_half(c[1], c[3], c[5], c[7]), 0x5410);
        if (KEYS) {
            const int token = 8 * upper + i;
            *reinterpret_cast<uint32_t *>(sm + (chunk >> 2) * 256 + token * 16 + (chunk & 3) * 4) = word;
            if (!(lane & 1)) sm[1024 + token * 8 + (chunk >> 1)] = (uint8_t)byte;
        } else {
            *reinterpret_cast<uint32_t *>(sm + (chunk * 8 + i) * 8 + upper * 4) = word;
            if (!upper) sm[1024 + chunk * 8 + i] = (uint8_t)byte;
        }
    }
    __syncwarp();
    uint8_t *const codes = dst + (KEYS ? 0 : kPackedV);
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4 *>(codes + (lane + 32 * i) * 16) = *reinterpret_cast<const uint4 *>(sm + (lane + 32 * i) * 16);
    if (lane < 8) *reinterpret_cast<uint4 *>(dst + (KEYS ? kPackedKScale : kPackedVScale) + lane * 16) = *reinterpret_cast<const uint4 *>(sm + 1024 + lane * 16);
}

// One layer's buffers, or several's (the parameters of a launch are sent with it: 48 bytes rather than 3 KiB where one will do).
template <int LAYERS>
struct PackLayers {
    const uint8_t *k_src[LAYERS];      // entries, or key blocks
    const uint8_t *v_src[LAYERS];
    const int32_t *src_table[LAYERS];  // [B][max_blocks] pages, or [B][Hkv][n_cols] slots
    const int32_t *block_table[LAYERS];
    uint8_t *packed[LAYERS];
    uint8_t *summaries[LAYERS];
};

// SLOTS: the source of block j is the entry of the local column that belongs to j, else of page src_table[b][j].
template <bool SLOTS, int LAYERS>
__global__ void __launch_bounds__(kPackWarps * 32)
pack_blocks_kernel(const __grid_constant__ PackLayers<LAYERS> ly, const int32_t *first_block, const int32_t *n_blocks,
                   int Hkv, int max_blocks, int max_new, int src_bytes, int n_cols, int local_col, uint32_t n_items, const Bounds bd)
{
    __shared__ __align__(16) uint8_t sm[kPackWarps][kPackedBytes / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = LAYERS == 1 ? 0 : blockIdx.y;
    const bool keys = warp < kPackWarps / 2;
    const uint32_t item = blockIdx.x * (kPackWarps / 2) + warp % (kPackWarps / 2);
    if (item >= n_items) return;
    const uint32_t steps = kPackTables.steps[lane];
    const float inverses = kPackTables.inverses[lane & 7];
    const uint32_t row = item / (uint32_t)Hkv;
    const int h = (int)(item % (uint32_t)Hkv), jj = (int)(row % (uint32_t)max_new), b = (int)(row / (uint32_t)max_new);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int n = n_blocks[b];
    const long long j = (long long)first_block[b] + jj;              // (both on their way at once)
    if (jj >= n) return;
    if (j < 0 || j >= max_blocks) {
        in_range(j, max_blocks, bd, kErrBlockCount);       // (checked build: reported; always skipped)
        return;
    }
    long long src;
    if (SLOTS) {
        src = ly.src_table[l][((long long)b * Hkv + h) * n_cols + local_col + (j & 1)];
        if (src < 0 || !in_range(src, bd.n_slots, bd, kErrSlot)) return;
    } else {
        src = (long long)ly.src_table[l][(long long)b * max_blocks + j] * Hkv + h;
        if (src_bytes == kEntryBytes && !in_range(src, bd.n_entries, bd, kErrHostEntry)) return;     // (a dense pool's extent is not declared)
    }
    const long long dst = (long long)ly.block_table[l][(long long)b * max_blocks + j] * Hkv + h;
    if (!in_range(dst, bd.n_entries, bd, kErrHostEntry)) return;
    const uint8_t *from = (keys ? ly.k_src[l] : ly.v_src[l]) + src * src_bytes + (lane >> 4) * 8 * kRowBytes + (lane & 15) * 16;
    uint32_t x[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 w = ld_once_v4(from + i * kRowBytes);
        x[i][0] = w.x; x[i][1] = w.y; x[i][2] = w.z; x[i][3] = w.w;
    }
    uint8_t *const entry = ly.packed[l] + dst * kPackedBytes;
    if (!keys) {
        pack_part<false>(x, steps, inverses, sm[warp], entry);
        return;
    }
    if (ly.summaries[l]) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            lo[p] = hi[p] = x[0][p];
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                lo[p] = bf2_min(lo[p], x[i][p]);
                hi[p] = bf2_max(hi[p], x[i][p]);
            }
            lo[p] = bf2_min(lo[p], __shfl_xor_sync(0xffffffffu, lo[p], 16));
            hi[p] = bf2_max(hi[p], __shfl_xor_sync(0xffffffffu, hi[p], 16));
        }
        uint8_t *const summary = ly.summaries[l] + (((long long)b * Hkv + h) * max_blocks + j) * kSummaryBytes;
        *reinterpret_cast<uint4 *>(summary + lane * 16) = lane < 16 ? make_uint4(lo[0], lo[1], lo[2], lo[3]) : make_uint4(hi[0], hi[1], hi[2], hi[3]);
    }
    pack_part<true>(x, steps, inverses, sm[warp], entry);
}

// One warp per list position: the packed entry through shared memory, the bf16 entry in sixteen 16-byte stores per lane.
__global__ void __launch_bounds__(kPackWarps * 32)
unpack_blocks_kernel(const uint8_t *packed, const long long *idx, int n, uint8_t *out, const Bounds bd)
{
    __shared__ __align__(16) uint8_t sm_all[kPackWarps][kPackedBytes];
    const int lane = threadIdx.x & 31, upper = lane >> 4, chunk = lane & 15;
    const long long item = (long long)blockIdx.x * kPackWarps + (threadIdx.x >> 5);
    if (item >= n) return;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long src = idx[item];
    if (src < 0 || !in_range(src, bd.n_entries, bd, kErrHostEntry)) return;
    uint8_t *sm = sm_all[threadIdx.x >> 5];
    const uint8_t *from = packed + src * kPackedBytes;
#pragma unroll
    for (int i = 0; i < 5; ++i)
        if (lane + 32 * i < kPackedBytes / 16) *reinterpret_cast<uint4 *>(sm + (lane + 32 * i) * 16) = ld_once_v4(from + (lane + 32 * i) * 16);
    __syncwarp();
    uint8_t *dst = out + item * kEntryBytes + upper * 8 * kRowBytes + chunk * 16;
    const uint32_t unit = 0x00010001u * ((127u + kDequantShift) << 7);          // (x, x) for 2^kDequantShift
    auto words = [&](uint32_t w, int byte, uint32_t (&o)[4]) {
        dequant_word(w, dequant_scale((uint32_t)byte * 0x00010001u), o);
#pragma unroll
        for (int p = 0; p < 4; ++p) o[p] = fma_bf16x2(o[p], unit, 0x80008000u);     // (-0 leaves a zero's sign as it is)
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int token = 8 * upper + i;
        uint32_t o[4];
        words(*reinterpret_cast<const uint32_t *>(sm + (chunk >> 2) * 256 + token * 16 + (chunk & 3) * 4), sm[kPackedKScale + token * 8 + (chunk >> 1)], o);
        *reinterpret_cast<uint4 *>(dst + i * kRowBytes) = make_uint4(o[0], o[1], o[2], o[3]);
    }
    // values: this lane's dims, eight tokens of each; then two dims of a token side by side
    uint32_t vals[8][4];                                             // [token][pair of dims]
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t o[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int dim = chunk * 8 + 2 * p + e;
            words(*reinterpret_cast<const uint32_t *>(sm + kPackedV + dim * 8 + upper * 4), sm[kPackedVScale + dim], o[e]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vals[2 * i][p] = __byte_perm(o[0][i], o[1][i], 0x5410);
            vals[2 * i + 1][p] = __byte_perm(o[0][i], o[1][i], 0x7632);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *reinterpret_cast<uint4 *>(dst + kPartBytes + i * kRowBytes) = make_uint4(vals[i][0], vals[i][1], vals[i][2], vals[i][3]);
}

// The checks and the launch that the three packing entry points share.
template <bool SLOTS, int LAYERS>
static int launch_pack(const char *who, const oasis_dims_t *dims, int n_layers, const PackLayers<LAYERS> &ly, const int32_t *first_block,
                       const int32_t *n_blocks, int max_new, int src_bytes, int n_cols, int local_col, void *stream)
{
    if (!first_block || !n_blocks) return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    if (max_new < 0 || max_new > dims->max_blocks)
        return fail(OASIS_ERR_INVALID_ARG, "%s: max_new_blocks %d outside [0, %d]", who, max_new, dims->max_blocks);
    for (int l = 0; l < n_layers; ++l) {
        if (!ly.k_src[l] || !ly.v_src[l] || !ly.src_table[l] || !ly.block_table[l] || !ly.packed[l])
            return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer (layer %d)", who, l);
        if (!aligned16(ly.k_src[l]) || !aligned16(ly.v_src[l]) || !aligned16(ly.packed[l]) || !aligned16(ly.summaries[l]))
            return fail(OASIS_ERR_INVALID_ARG, "%s: pools and summaries must be 16-byte aligned (layer %d)", who, l);
    }
    const long long n_items = (long long)dims->batch * dims->n_kv_heads * max_new;
    if (n_items == 0 || n_layers == 0) return OASIS_OK;
    if (n_items > 0x7fffffffLL) return fail(OASIS_ERR_UNSUPPORTED, "%s: too many blocks", who);
    const long long grid = (n_items + kPackWarps / 2 - 1) / (kPackWarps / 2);
    prefer_max_shared_carveout(pack_blocks_kernel<SLOTS, LAYERS>);
    const cudaError_t e = launch_waiting(pack_blocks_kernel<SLOTS, LAYERS>, dim3((unsigned)grid, (unsigned)n_layers), kPackWarps * 32, (cudaStream_t)stream, ly,
                                         first_block, n_blocks, (int)dims->n_kv_heads, (int)dims->max_blocks, max_new, src_bytes, n_cols, local_col,
                                         (uint32_t)n_items, bounds());
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    return OASIS_OK;
}

}  // namespace oasis

extern "C" int oasis_pack_blocks(const oasis_dims_t *dims, const void *kv_pool, const int32_t *src_table, const int32_t *first_block,
                                 const int32_t *n_blocks, int32_t max_new_blocks, void *packed, const int32_t *block_table,
                                 void *summaries, void *stream)
{
    using namespace oasis;
    if (int rc = check_dims(dims)) return rc;
    PackLayers<1> ly = {};
    ly.k_src[0] = (const uint8_t *)kv_pool;
    ly.v_src[0] = kv_pool ? (const uint8_t *)kv_pool + kPartBytes : nullptr;
    ly.src_table[0] = src_table;
    ly.block_table[0] = block_table;
    ly.packed[0] = (uint8_t *)packed;
    ly.summaries[0] = (uint8_t *)summaries;
    return launch_pack<false>("oasis_pack_blocks", dims, 1, ly, first_block, n_blocks, max_new_blocks, kEntryBytes, 0, 0, stream);
}

extern "C" int oasis_offload_blocks_packed(const oasis_dims_t *dims, const void *dense_k, const void *dense_v, const int32_t *gpu_table,
                                           const int32_t *block_table, const int32_t *first_block, const int32_t *n_blocks,
                                           int32_t max_new_blocks, void *packed, void *summaries, void *stream)
{
    using namespace oasis;
    if (int rc = check_dims(dims)) return rc;
    PackLayers<1> ly = {};
    ly.k_src[0] = (const uint8_t *)dense_k;
    ly.v_src[0] = (const uint8_t *)dense_v;
    ly.src_table[0] = gpu_table;
    ly.block_table[0] = block_table;
    ly.packed[0] = (uint8_t *)packed;
    ly.summaries[0] = (uint8_t *)summaries;
    return launch_pack<false>("oasis_offload_blocks_packed", dims, 1, ly, first_block, n_blocks, max_new_blocks, kPartBytes, 0, 0, stream);
}

extern "C" int oasis_pack_local_layers(const oasis_dims_t *dims, int32_t n_layers, const void *const *hbm_pools,
                                       const int32_t *const *slot_tbls, int32_t n_cols, int32_t local_col, const int32_t *first_block,
                                       const int32_t *n_blocks, int32_t max_new_blocks, void *const *packed,
                                       const int32_t *const *block_tables, void *const *summaries, void *stream)
{
    using namespace oasis;
    const char *who = "oasis_pack_local_layers";
    if (int rc = check_dims(dims)) return rc;
    if (n_layers < 0 || n_layers > OASIS_MAX_APPEND_LAYERS)
        return fail(OASIS_ERR_INVALID_ARG, "%s: n_layers %d outside [0, %d]", who, n_layers, OASIS_MAX_APPEND_LAYERS);
    if (n_cols < 2 || local_col < 0 || local_col > n_cols - 2)
        return fail(OASIS_ERR_INVALID_ARG, "%s: local_col %d, n_cols %d", who, local_col, n_cols);
    if (max_new_blocks > 2)
        return fail(OASIS_ERR_INVALID_ARG, "%s: max_new_blocks %d: the local window holds two blocks", who, max_new_blocks);
    if (n_layers == 0) return OASIS_OK;
    if (!hbm_pools || !slot_tbls || !packed || !block_tables) return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    PackLayers<OASIS_MAX_APPEND_LAYERS> ly = {};
    for (int l = 0; l < n_layers; ++l) {
        ly.k_src[l] = (const uint8_t *)hbm_pools[l];
        ly.v_src[l] = hbm_pools[l] ? (const uint8_t *)hbm_pools[l] + kPartBytes : nullptr;
        ly.src_table[l] = slot_tbls[l];
        ly.block_table[l] = block_tables[l];
        ly.packed[l] = (uint8_t *)packed[l];
        ly.summaries[l] = summaries ? (uint8_t *)summaries[l] : nullptr;
    }
    return launch_pack<true>(who, dims, n_layers, ly, first_block, n_blocks, max_new_blocks, kEntryBytes, n_cols, local_col, stream);
}

extern "C" int oasis_unpack_blocks(const void *packed, const int64_t *idx, int32_t n, void *out, void *stream)
{
    using namespace oasis;
    const char *who = "oasis_unpack_blocks";
    if (n < 0) return fail(OASIS_ERR_INVALID_ARG, "%s: n %d < 0", who, n);
    if (n == 0) return OASIS_OK;
    if (!packed || !idx || !out) return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    if (!aligned16(packed) || !aligned16(out)) return fail(OASIS_ERR_INVALID_ARG, "%s: packed and out must be 16-byte aligned", who);
    prefer_max_shared_carveout(unpack_blocks_kernel);
    const cudaError_t e = launch_waiting(unpack_blocks_kernel, dim3((unsigned)((n - 1) / kPackWarps + 1)), kPackWarps * 32, (cudaStream_t)stream,
                                         (const uint8_t *)packed, (const long long *)idx, (int)n, (uint8_t *)out, bounds());
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    return OASIS_OK;
}
