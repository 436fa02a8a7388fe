// Commit of a verified path of a draft tree: the kept nodes' keys and values go from the step's tree buffer into the
// local window of the working set and into the CPU full-KV pool, for all layers in one launch.
//
// One warp per (layer, request, KV head): lanes 0-15 carry 256-byte key rows, lanes 16-31 the value rows, 16 bytes each.  The
// length, the count, the path and the two blocks' places are read once per warp, in two rounds of loads (lane i holds path
// entry i; lanes 0 and 1 the places of the even and the odd block), then up to eight rows are in flight at a time.
// Traffic per layer: 512 B read and 2 x 512 B written per (request, kept token, head).  A warp per row, which read all of that
// for each of them, took 9.2 us for 32 layers of 16 requests x 8 heads x 4 tokens (28 MB); this 6.0 us (0.71 of the copy rate) with the
// full-KV pool in HBM.  Into pinned host memory the link bounds it: 190 us, 49 GB/s (a copy takes 57).  The launch may
// overlap the end of the previous kernel, for which every warp waits before its first load (8.3 -> 6.0 us a call, launched one
// by one); letting its own successor start early costs more than it gains (7.2 instead of 6.4 us for 549 thread blocks).
#include "common.cuh"

namespace oasis {

constexpr int kCommitWarps = 4, kCommitRows = 8;

struct CommitLayers {
    const uint8_t *tree_kv[OASIS_MAX_APPEND_LAYERS];
    const int32_t *block_table[OASIS_MAX_APPEND_LAYERS];
    const int32_t *slot_tbl[OASIS_MAX_APPEND_LAYERS];
    int32_t *blk_tbl[OASIS_MAX_APPEND_LAYERS];
    uint8_t *pool[OASIS_MAX_APPEND_LAYERS];
    uint8_t *host_kv[OASIS_MAX_APPEND_LAYERS];
};

struct CommitParams {
    const int32_t *path, *n_commit, *seq_len, *n_candidates;
    int32_t *next_len;
    int B, T, M, Hkv, max_blocks, n_cols, local_col;
};

__global__ void __launch_bounds__(kCommitWarps * 32)
commit_kv_kernel(const __grid_constant__ CommitLayers ly, const CommitParams p, const Bounds bd)
{
    const int l = blockIdx.y, lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * kCommitWarps + (threadIdx.x >> 5);     // (request, head)
    if (row >= (long long)p.B * p.Hkv) return;
    const int b = (int)(row / p.Hkv), h = (int)(row % p.Hkv);
    asm volatile("griddepcontrol.wait;" ::: "memory");              // (the launch may overlap the end of the previous kernel)
    const int n_raw = p.n_commit[b], L = p.seq_len[b], n_cand = p.n_candidates ? p.n_candidates[b] : 0;
    const int t_mine = lane < p.M ? p.path[b * p.M + lane] : -1;
    const int n = max(0, min(n_raw, p.M));
    if (p.next_len && l == 0 && h == 0 && lane == 0) p.next_len[b] = L + n;
    if (n == 0 && lane < 2) {                                        // a local block that may have been selected leaves its column
        int32_t *const col = ly.blk_tbl[l] + row * p.n_cols + p.local_col + lane;
        if (n_cand > 0 && *col >= 0 && *col < n_cand) *col = -1;
    }
    if (n == 0 || L < 0) return;
    const int lo = L / kBlock, hi = (L + n - 1) / kBlock;
    // lane 0: block lo, lane 1: the next one; their slot and their entry of the full-KV pool, -1 where there is none
    long long slot = -1, entry = -1;
    if (lane < 2) {
        const int j = lo + lane;
        if (j <= hi && j < p.max_blocks) {
            slot = ly.slot_tbl[l][row * p.n_cols + p.local_col + (j & 1)];
            if (slot >= 0 && !in_range(slot, bd.n_slots, bd, kErrSlot)) slot = -1;
            if (ly.host_kv[l]) {
                const long long phys = ly.block_table[l][(long long)b * p.max_blocks + j];
                entry = phys * p.Hkv + h;
                if (phys < 0 || !in_range(entry, bd.n_entries, bd, kErrHostEntry)) entry = -1;
            }
        } else if (kBoundsCheck && j <= hi) {
            in_range(j, p.max_blocks, bd, kErrBlockId);
        }
        ly.blk_tbl[l][row * p.n_cols + p.local_col + (j & 1)] = j <= hi ? j : -1;
    }
    const long long slot0 = __shfl_sync(0xffffffffu, slot, 0), slot1 = __shfl_sync(0xffffffffu, slot, 1);
    const long long entry0 = __shfl_sync(0xffffffffu, entry, 0), entry1 = __shfl_sync(0xffffffffu, entry, 1);
    const int part = lane >> 4, off = (lane & 15) * 16;                      // 0: key row, 1: value row
    const uint8_t *src = ly.tree_kv[l] + ((long long)b * p.T * p.Hkv + h) * 2 * kRowBytes + part * kRowBytes + off;
    uint8_t *const pool = ly.pool[l] + part * kPartBytes + off, *const host = ly.host_kv[l] + part * kPartBytes + off;
    for (int i0 = 0; i0 < n; i0 += kCommitRows) {
        uint4 v[kCommitRows];
        bool ok[kCommitRows];
#pragma unroll
        for (int k = 0; k < kCommitRows; ++k) {
            const int t = __shfl_sync(0xffffffffu, t_mine, (i0 + k) & 31);
            ok[k] = i0 + k < n && t >= 0 && t < p.T;
            if (ok[k]) v[k] = *reinterpret_cast<const uint4 *>(src + (long long)t * p.Hkv * 2 * kRowBytes);
        }
#pragma unroll
        for (int k = 0; k < kCommitRows; ++k) {
            const int pos = L + i0 + k;
            const long long s = pos / kBlock == lo ? slot0 : slot1, e = pos / kBlock == lo ? entry0 : entry1;
            if (ok[k] && s >= 0) *reinterpret_cast<uint4 *>(pool + s * kEntryBytes + pos % kBlock * kRowBytes) = v[k];
            if (ok[k] && e >= 0) *reinterpret_cast<uint4 *>(host + e * kEntryBytes + pos % kBlock * kRowBytes) = v[k];
        }
    }
}

static int launch_commit(const oasis_dims_t *dims, int n_layers, const void *const *tree_kvs, int T, const int32_t *path,
                         int M, const int32_t *n_commit, const int32_t *seq_len, const int32_t *const *block_tables,
                         const int32_t *const *slot_tbls, int32_t *const *blk_tbls, int n_cols, int local_col,
                         void *const *pools, void *const *host_kvs, const int32_t *n_candidates, int32_t *next_len, cudaStream_t st,
                         const char *who)
{
    if (int rc = check_dims(dims)) return rc;
    if (n_layers < 0 || n_layers > OASIS_MAX_APPEND_LAYERS)
        return fail(OASIS_ERR_INVALID_ARG, "%s: n_layers %d outside [0, %d]", who, n_layers, OASIS_MAX_APPEND_LAYERS);
    if (T < 1 || T > OASIS_MAX_TREE)
        return fail(OASIS_ERR_INVALID_ARG, "%s: n_tree %d outside [1, %d]", who, T, OASIS_MAX_TREE);
    if (M < 1 || M > kBlock) return fail(OASIS_ERR_INVALID_ARG, "%s: max_path %d outside [1, %d]", who, M, kBlock);
    if (local_col < 0 || n_cols < 2 || local_col > n_cols - 2)
        return fail(OASIS_ERR_INVALID_ARG, "%s: local columns %d and the next one outside the %d columns", who, local_col, n_cols);
    if (dims->batch == 0 || n_layers == 0) return OASIS_OK;
    if (!tree_kvs || !path || !n_commit || !seq_len || !block_tables || !slot_tbls || !blk_tbls || !pools)
        return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    const auto overlaps = [&](const int32_t *in, long long n) {        // (all layers and heads read them, in no order)
        const uintptr_t a = reinterpret_cast<uintptr_t>(next_len), c = reinterpret_cast<uintptr_t>(in);
        return a < c + 4 * (uintptr_t)n && c < a + 4 * (uintptr_t)dims->batch;
    };
    if (next_len && (overlaps(seq_len, dims->batch) || overlaps(n_commit, dims->batch) || overlaps(path, (long long)dims->batch * M) ||
                     (n_candidates && overlaps(n_candidates, dims->batch))))
        return fail(OASIS_ERR_INVALID_ARG, "%s: next_len may not share memory with seq_len, n_commit, path or n_candidates", who);
    CommitLayers ly = {};
    for (int l = 0; l < n_layers; ++l) {
        void *host = host_kvs ? host_kvs[l] : nullptr;
        if (!tree_kvs[l] || !slot_tbls[l] || !blk_tbls[l] || !pools[l] || (host && !block_tables[l]))
            return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer for layer %d", who, l);
        if (!aligned16(tree_kvs[l]) || !aligned16(pools[l]) || !aligned16(host))
            return fail(OASIS_ERR_INVALID_ARG, "%s: tree_kv, hbm_pool and host_kv must be 16-byte aligned (layer %d)", who, l);
        ly.tree_kv[l] = (const uint8_t *)tree_kvs[l];
        ly.block_table[l] = block_tables[l];
        ly.slot_tbl[l] = slot_tbls[l];
        ly.blk_tbl[l] = blk_tbls[l];
        ly.pool[l] = (uint8_t *)pools[l];
        ly.host_kv[l] = (uint8_t *)host;
    }
    const long long total = (long long)dims->batch * dims->n_kv_heads;
    CommitParams p;
    p.path = path; p.n_commit = n_commit; p.seq_len = seq_len; p.next_len = next_len; p.n_candidates = n_candidates;
    p.B = dims->batch; p.T = T; p.M = M; p.Hkv = dims->n_kv_heads; p.max_blocks = dims->max_blocks;
    p.n_cols = n_cols; p.local_col = local_col;
    prefer_max_shared_carveout(commit_kv_kernel);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((total + kCommitWarps - 1) / kCommitWarps), (unsigned)n_layers);
    cfg.blockDim = dim3(kCommitWarps * 32);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, commit_kv_kernel, ly, p, bounds());
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    return OASIS_OK;
}

}  // namespace oasis

extern "C" int oasis_commit_kv(const oasis_dims_t *dims, const void *tree_kv, int32_t n_tree, const int32_t *path,
                               int32_t max_path, const int32_t *n_commit, const int32_t *seq_len,
                               const int32_t *block_table, const int32_t *slot_tbl, int32_t *blk_tbl, int32_t n_cols,
                               int32_t local_col, void *hbm_pool, void *host_kv, int32_t *next_len, void *stream)
{
    return oasis::launch_commit(dims, 1, &tree_kv, n_tree, path, max_path, n_commit, seq_len, &block_table, &slot_tbl, &blk_tbl,
                                n_cols, local_col, &hbm_pool, &host_kv, nullptr, next_len, (cudaStream_t)stream, "oasis_commit_kv");
}

extern "C" int oasis_commit_kv_layers(const oasis_dims_t *dims, int32_t n_layers, const void *const *tree_kvs, int32_t n_tree,
                                      const int32_t *path, int32_t max_path, const int32_t *n_commit, const int32_t *seq_len,
                                      const int32_t *const *block_tables, const int32_t *const *slot_tbls,
                                      int32_t *const *blk_tbls, int32_t n_cols, int32_t local_col, void *const *hbm_pools,
                                      void *const *host_kvs, int32_t *next_len, void *stream)
{
    return oasis::launch_commit(dims, n_layers, tree_kvs, n_tree, path, max_path, n_commit, seq_len, block_tables, slot_tbls,
                                blk_tbls, n_cols, local_col, hbm_pools, host_kvs, nullptr, next_len, (cudaStream_t)stream,
                                "oasis_commit_kv_layers");
}

extern "C" int oasis_commit_kv_layers_after_select(const oasis_dims_t *dims, int32_t n_layers, const void *const *tree_kvs, int32_t n_tree,
                                                   const int32_t *path, int32_t max_path, const int32_t *n_commit, const int32_t *seq_len,
                                                   const int32_t *const *block_tables, const int32_t *const *slot_tbls,
                                                   int32_t *const *blk_tbls, int32_t n_cols, int32_t local_col, void *const *hbm_pools,
                                                   void *const *host_kvs, const int32_t *n_candidates, int32_t *next_len, void *stream)
{
    return oasis::launch_commit(dims, n_layers, tree_kvs, n_tree, path, max_path, n_commit, seq_len, block_tables, slot_tbls,
                                blk_tbls, n_cols, local_col, hbm_pools, host_kvs, n_candidates, next_len, (cudaStream_t)stream,
                                "oasis_commit_kv_layers_after_select");
}
