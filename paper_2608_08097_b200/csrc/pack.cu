// Blocks of the KV cache in 4 bits: packing (from entries of a pool, from the local window, from a dense pool's separate key and
// value blocks) and unpacking.  The format and its arithmetic are in packed.cuh.
//
// Packing: one warp per (request, block, KV head).  Sixteen 16-byte loads per lane bring the 8 KiB of keys and values, each
// warp-wide load two 256-byte token rows: a lane holds the same eight dims of eight tokens, even ones in lanes 0..15 and odd ones
// in lanes 16..31.  The largest magnitude of a key's group (16 dims of a token) is one exchange with the neighbouring lane away, of
// a value's group (16 tokens of a dim) seven maxima and one exchange with the other half-warp.  The lane's eight codes of a key
// are one word.  The entry is put together in shared memory and leaves in 16-byte stores, whole lines, because its place is
// usually in pinned host memory.  The block's summaries (minimum and maximum of the keys) come from the same registers.
// Algorithmic traffic: 8,192 B read, 2,304 B (and 512 B of summaries) written per (block, head).
#include "packed.cuh"

namespace oasis {

constexpr int kPackWarps = 4;

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
// NaN counts as zero.
__device__ __forceinline__ uint32_t without_nan(uint32_t v)
{
    const uint32_t lo = (v & 0x7fffu) > 0x7f80u ? 0u : v & 0xffffu, hi = (v & 0x7fff0000u) > 0x7f800000u ? 0u : v & 0xffff0000u;
    return lo | hi;
}
__device__ __forceinline__ bool has_nan(uint32_t v) { return (v & 0x7fffu) > 0x7f80u || (v & 0x7fff0000u) > 0x7f800000u; }

// keys (k) and values (v) of one block and head, lane -> 16-byte chunk (lane & 15) of token (lane >> 4) + 2 i; `sm`: 2,304 bytes
// of this warp, 16-byte aligned; `dst`: the packed entry; `summary` (or NULL): its 512 bytes.
__device__ __forceinline__ void pack_entry(uint32_t (&k)[8][4], uint32_t (&v)[8][4], uint8_t *sm, uint8_t *dst, uint8_t *summary)
{
    const int lane = threadIdx.x & 31, odd = lane >> 4, chunk = lane & 15;
    if (summary) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            lo[p] = hi[p] = k[0][p];
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                lo[p] = bf2_min(lo[p], k[i][p]);
                hi[p] = bf2_max(hi[p], k[i][p]);
            }
            lo[p] = bf2_min(lo[p], __shfl_xor_sync(0xffffffffu, lo[p], 16));
            hi[p] = bf2_max(hi[p], __shfl_xor_sync(0xffffffffu, hi[p], 16));
        }
        *reinterpret_cast<uint4 *>(summary + lane * 16) =
            odd ? make_uint4(hi[0], hi[1], hi[2], hi[3]) : make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int p = 0; p < 4; ++p) nan |= has_nan(k[i][p]) | has_nan(v[i][p]);
    if (__any_sync(0xffffffffu, nan)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                k[i][p] = without_nan(k[i][p]);
                v[i][p] = without_nan(v[i][p]);
            }
    }
    // keys: two lanes per group
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t a2 = bf2_max(bf2_max(k[i][0] & 0x7fff7fffu, k[i][1] & 0x7fff7fffu), bf2_max(k[i][2] & 0x7fff7fffu, k[i][3] & 0x7fff7fffu));
        a2 = bf2_max(a2, __shfl_xor_sync(0xffffffffu, a2, 1));
        const int byte = scale_byte(fmaxf(bf_lo(a2), bf_hi(a2)));
        const float inv = scale_inverse(byte);
        uint32_t w = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) w |= (code_bits(bf_lo(k[i][p]), inv) | code_bits(bf_hi(k[i][p]), inv) << 16) << (4 * p);
        const int token = odd + 2 * i;
        *reinterpret_cast<uint32_t *>(sm + (chunk >> 2) * 256 + token * 16 + (chunk & 3) * 4) = w;
        if (!(lane & 1)) sm[kPackedKScale + token * 8 + (chunk >> 1)] = (uint8_t)byte;
    }
    // values: the lane's eight dims, its tokens in the low (even) or high (odd) halves of the words
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t a2 = v[0][p] & 0x7fff7fffu;
#pragma unroll
        for (int i = 1; i < 8; ++i) a2 = bf2_max(a2, v[i][p] & 0x7fff7fffu);
        a2 = bf2_max(a2, __shfl_xor_sync(0xffffffffu, a2, 16));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int dim = chunk * 8 + 2 * p + e;
            const int byte = scale_byte(e ? bf_hi(a2) : bf_lo(a2));
            const float inv = scale_inverse(byte);
            uint32_t half[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) half[i >> 2] |= code_bits(e ? bf_hi(v[i][p]) : bf_lo(v[i][p]), inv) << (4 * (i & 3));
#pragma unroll
            for (int w = 0; w < 2; ++w) *reinterpret_cast<uint16_t *>(sm + kPackedV + dim * 8 + w * 4 + odd * 2) = (uint16_t)half[w];
            if (!odd) sm[kPackedVScale + dim] = (uint8_t)byte;
        }
    }
    __syncwarp();
#pragma unroll
    for (int i = lane; i < kPackedBytes / 16; i += 32) *reinterpret_cast<uint4 *>(dst + i * 16) = *reinterpret_cast<const uint4 *>(sm + i * 16);
}

struct PackLayers {
    const uint8_t *k_src[OASIS_MAX_APPEND_LAYERS];      // entries, or key blocks
    const uint8_t *v_src[OASIS_MAX_APPEND_LAYERS];
    const int32_t *src_table[OASIS_MAX_APPEND_LAYERS];  // [B][max_blocks] pages, or [B][Hkv][n_cols] slots
    const int32_t *block_table[OASIS_MAX_APPEND_LAYERS];
    uint8_t *packed[OASIS_MAX_APPEND_LAYERS];
    uint8_t *summaries[OASIS_MAX_APPEND_LAYERS];
};

// SLOTS: the source of block j is the entry of the local column that belongs to j, else of page src_table[b][j].
template <bool SLOTS>
__global__ void __launch_bounds__(kPackWarps * 32)
pack_blocks_kernel(const __grid_constant__ PackLayers ly, const int32_t *__restrict__ first_block, const int32_t *__restrict__ n_blocks,
                   int Hkv, int max_blocks, int max_new, int src_bytes, int n_cols, int local_col, long long n_items, const Bounds bd)
{
    __shared__ __align__(16) uint8_t sm[kPackWarps][kPackedBytes];
    const int lane = threadIdx.x & 31, l = blockIdx.y;
    const long long item = (long long)blockIdx.x * kPackWarps + (threadIdx.x >> 5);
    if (item >= n_items) return;
    const int h = (int)(item % Hkv);
    const int jj = (int)((item / Hkv) % max_new);
    const int b = (int)(item / ((long long)Hkv * max_new));
    if (jj >= n_blocks[b]) return;
    const long long j = (long long)first_block[b] + jj;
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
    }
    const long long dst = (long long)ly.block_table[l][(long long)b * max_blocks + j] * Hkv + h;
    if (!in_range(dst, bd.n_entries, bd, kErrHostEntry)) return;
    const uint8_t *ksrc = ly.k_src[l] + src * src_bytes + lane * 16, *vsrc = ly.v_src[l] + src * src_bytes + lane * 16;
    uint32_t k[8][4], v[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 w = ld_stream_v4(ksrc + i * 512);
        k[i][0] = w.x; k[i][1] = w.y; k[i][2] = w.z; k[i][3] = w.w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 w = ld_stream_v4(vsrc + i * 512);
        v[i][0] = w.x; v[i][1] = w.y; v[i][2] = w.z; v[i][3] = w.w;
    }
    pack_entry(k, v, sm[threadIdx.x >> 5], ly.packed[l] + dst * kPackedBytes,
               ly.summaries[l] ? ly.summaries[l] + (((long long)b * Hkv + h) * max_blocks + j) * kSummaryBytes : nullptr);
}

// One warp per list position: the packed entry through shared memory, the bf16 entry in sixteen 16-byte stores per lane.
__global__ void __launch_bounds__(kPackWarps * 32)
unpack_blocks_kernel(const uint8_t *__restrict__ packed, const long long *__restrict__ idx, int n, uint8_t *__restrict__ out, const Bounds bd)
{
    __shared__ __align__(16) uint8_t sm_all[kPackWarps][kPackedBytes];
    const int lane = threadIdx.x & 31, odd = lane >> 4, chunk = lane & 15;
    const long long item = (long long)blockIdx.x * kPackWarps + (threadIdx.x >> 5);
    if (item >= n) return;
    const long long src = idx[item];
    if (src < 0 || !in_range(src, bd.n_entries, bd, kErrHostEntry)) return;
    uint8_t *sm = sm_all[threadIdx.x >> 5];
    const uint8_t *from = packed + src * kPackedBytes;
#pragma unroll
    for (int i = 0; i < 5; ++i)
        if (lane + 32 * i < kPackedBytes / 16) *reinterpret_cast<uint4 *>(sm + (lane + 32 * i) * 16) = ld_stream_v4(from + (lane + 32 * i) * 16);
    __syncwarp();
    uint8_t *dst = out + item * kEntryBytes + lane * 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int token = odd + 2 * i;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(sm + (chunk >> 2) * 256 + token * 16 + (chunk & 3) * 4);
        const float sc = scale_value(sm[kPackedKScale + token * 8 + (chunk >> 1)]);
        uint32_t o[4];
#pragma unroll
        for (int p = 0; p < 4; ++p)
            o[p] = pack_bf16x2((float)((int)((w >> (4 * p)) & 15u) - 8) * sc, (float)((int)((w >> (16 + 4 * p)) & 15u) - 8) * sc);
        *reinterpret_cast<uint4 *>(dst + i * 512) = make_uint4(o[0], o[1], o[2], o[3]);
    }
    // values: this lane's dims, both words of each; token 2 i + odd of word i >> 2 is in place i & 3 of its half of the word
    uint32_t vals[8][4];                                             // [i][pair of dims]
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        float s[2];
        uint32_t w[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int dim = chunk * 8 + 2 * p + e;
            s[e] = scale_value(sm[kPackedVScale + dim]);
            const uint2 both = *reinterpret_cast<const uint2 *>(sm + kPackedV + dim * 8);
            w[e][0] = both.x >> (16 * odd);
            w[e][1] = both.y >> (16 * odd);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float lo = (float)((int)((w[0][i >> 2] >> (4 * (i & 3))) & 15u) - 8) * s[0];
            const float hi = (float)((int)((w[1][i >> 2] >> (4 * (i & 3))) & 15u) - 8) * s[1];
            vals[i][p] = pack_bf16x2(lo, hi);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *reinterpret_cast<uint4 *>(dst + kPartBytes + i * 512) = make_uint4(vals[i][0], vals[i][1], vals[i][2], vals[i][3]);
}

// The checks and the launch that the three packing entry points share.
static int launch_pack(const char *who, const oasis_dims_t *dims, int n_layers, const PackLayers &ly, bool slots, const int32_t *first_block,
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
    const long long grid = (n_items + kPackWarps - 1) / kPackWarps;
    if (grid > 0x7fffffffLL) return fail(OASIS_ERR_UNSUPPORTED, "%s: too many blocks", who);
    const dim3 g((unsigned)grid, (unsigned)n_layers);
    if (slots) {
        prefer_max_shared_carveout(pack_blocks_kernel<true>);
        pack_blocks_kernel<true><<<g, kPackWarps * 32, 0, (cudaStream_t)stream>>>(ly, first_block, n_blocks, dims->n_kv_heads, dims->max_blocks,
                                                                                  max_new, src_bytes, n_cols, local_col, n_items, bounds());
    } else {
        prefer_max_shared_carveout(pack_blocks_kernel<false>);
        pack_blocks_kernel<false><<<g, kPackWarps * 32, 0, (cudaStream_t)stream>>>(ly, first_block, n_blocks, dims->n_kv_heads, dims->max_blocks,
                                                                                   max_new, src_bytes, n_cols, local_col, n_items, bounds());
    }
    return check_launch(who);
}

}  // namespace oasis

extern "C" int oasis_pack_blocks(const oasis_dims_t *dims, const void *kv_pool, const int32_t *src_table, const int32_t *first_block,
                                 const int32_t *n_blocks, int32_t max_new_blocks, void *packed, const int32_t *block_table,
                                 void *summaries, void *stream)
{
    using namespace oasis;
    if (int rc = check_dims(dims)) return rc;
    PackLayers ly = {};
    ly.k_src[0] = (const uint8_t *)kv_pool;
    ly.v_src[0] = kv_pool ? (const uint8_t *)kv_pool + kPartBytes : nullptr;
    ly.src_table[0] = src_table;
    ly.block_table[0] = block_table;
    ly.packed[0] = (uint8_t *)packed;
    ly.summaries[0] = (uint8_t *)summaries;
    return launch_pack("oasis_pack_blocks", dims, 1, ly, false, first_block, n_blocks, max_new_blocks, kEntryBytes, 0, 0, stream);
}

extern "C" int oasis_offload_blocks_packed(const oasis_dims_t *dims, const void *dense_k, const void *dense_v, const int32_t *gpu_table,
                                           const int32_t *block_table, const int32_t *first_block, const int32_t *n_blocks,
                                           int32_t max_new_blocks, void *packed, void *summaries, void *stream)
{
    using namespace oasis;
    if (int rc = check_dims(dims)) return rc;
    PackLayers ly = {};
    ly.k_src[0] = (const uint8_t *)dense_k;
    ly.v_src[0] = (const uint8_t *)dense_v;
    ly.src_table[0] = gpu_table;
    ly.block_table[0] = block_table;
    ly.packed[0] = (uint8_t *)packed;
    ly.summaries[0] = (uint8_t *)summaries;
    return launch_pack("oasis_offload_blocks_packed", dims, 1, ly, false, first_block, n_blocks, max_new_blocks, kPartBytes, 0, 0, stream);
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
    PackLayers ly = {};
    for (int l = 0; l < n_layers; ++l) {
        ly.k_src[l] = (const uint8_t *)hbm_pools[l];
        ly.v_src[l] = hbm_pools[l] ? (const uint8_t *)hbm_pools[l] + kPartBytes : nullptr;
        ly.src_table[l] = slot_tbls[l];
        ly.block_table[l] = block_tables[l];
        ly.packed[l] = (uint8_t *)packed[l];
        ly.summaries[l] = summaries ? (uint8_t *)summaries[l] : nullptr;
    }
    return launch_pack(who, dims, n_layers, ly, true, first_block, n_blocks, max_new_blocks, kEntryBytes, n_cols, local_col, stream);
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
    unpack_blocks_kernel<<<(n - 1) / kPackWarps + 1, kPackWarps * 32, 0, (cudaStream_t)stream>>>(
        (const uint8_t *)packed, (const long long *)idx, n, (uint8_t *)out, bounds());
    return check_launch(who);
}
