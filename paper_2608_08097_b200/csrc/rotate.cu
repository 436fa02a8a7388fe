// Rotary positions of a step's (or a prompt's) projections: qkv rows in, rotated queries and the keys' and values' rows out, in the
// layouts that the attention and the KV append read.
//
//   y_i = m (x_i cos a - x_i' sin a),   y_i' = m (x_i' cos a + x_i sin a),   a = position * frequency_i
// over the first rot_dim dims of queries and keys (i' = i + rot_dim / 2, or pairs side by side); what lies behind them and the
// values are copied.  Angles: the position times the frequency in turns (frequency / 2 pi), in 64 bits, of which only the fraction
// of a turn is kept, exactly, before anything is rounded to fp32: a position of a million loses nothing.
// A thread block takes one or a few tokens: its threads work out their cosines and sines once, into shared memory, and then a
// half-warp moves a head's row at a time, 8 dims a lane; the first rows are on their way before the angles.  With halves the partner's
// dims come from another lane of the half-warp, or, where the half is no multiple of 8, through shared memory (a row of fp32, a word
// of padding after every eight).  Every element is read once and written once.
// In a draft tree a token's position is seq_len + its depth, which one warp finds by pointer doubling over the parents.
// Bound by HBM: 8,192 tokens of 32 + 8 + 8 heads in bf16 35.5 us (201 MB, 5.7 TB/s).  3,003 tokens of 20 + 4 + 4 heads in fp32 with
// halves of 26 dims 15.8 us (65 MB, 4.1 TB/s; 33 us when every lane gathered its partners from global memory).  One token: 2.8 us,
// a launch.
#include "common.cuh"

namespace oasis {

constexpr int kRotThreads = 128, kRotLanes = 16, kRotWorkers = kRotThreads / kRotLanes;
constexpr int kRotMaxTokens = 8;                            // tokens of a thread block at most

struct RotateParams {
    const uint8_t *qkv;
    const int32_t *positions, *seq_len, *parent, *n_nodes;
    const double *freqs;
    uint8_t *q, *kv;
    long long batch_stride, token_stride;                   // elements
    int T, Hq, Hkv, rot, tokens_per_block;
    long long n_tokens;
    float factor;
};

// 8 elements in W 32-bit registers as floats.
template <int TYPE, int W>
__device__ __forceinline__ void to_floats(const uint32_t (&w)[W], float (&x)[8])
{
    if constexpr (TYPE == OASIS_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
    } else if constexpr (TYPE == OASIS_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[e]));
            x[2 * e] = f.x;
            x[2 * e + 1] = f.y;
        }
    }
}

enum { kSideBySide = 0, kHalves = 1, kOddHalves = 2 };      // pairs; halves of a multiple of 8 dims; other halves

template <int TYPE, int MODE>
__global__ void __launch_bounds__(kRotThreads)
rotate_qkv_kernel(const RotateParams p)
{
    constexpr int SIZE = TYPE == OASIS_F32 ? 4 : 2, W = 2 * SIZE;        // registers of 8 elements
    constexpr int AHEAD = TYPE == OASIS_F32 ? 2 : 3;                     // rows of a half-warp in flight
    __shared__ __align__(16) float2 turn[kRotMaxTokens][kHeadDim / 2];   // (cos, sin) times the factor
    __shared__ int s_depth[kRotMaxTokens];
    __shared__ float s_row[MODE == kOddHalves ? kRotWorkers : 1][kRotLanes * 9];
    const int tid = threadIdx.x, lane = tid & 31;
    const uint32_t n0 = blockIdx.x * (uint32_t)p.tokens_per_block, T = (uint32_t)p.T;     // (at most 2^31 tokens)
    const int here = (int)min((uint32_t)p.tokens_per_block, (uint32_t)p.n_tokens - n0);
    const int worker = tid / kRotLanes, chunk = tid % kRotLanes, d0 = chunk * 8;
    const int n_rot = p.Hq + p.Hkv, n_rows = p.Hq + 2 * p.Hkv;
    uint32_t w[AHEAD][W];
    auto load = [&](int k, int a0) {                                     // rows a0, a0 + kRotWorkers, .. of token n0 + k
        const uint32_t n = n0 + k;
        const uint8_t *src = p.qkv + ((long long)(n / T) * p.batch_stride + (long long)(n % T) * p.token_stride + d0) * SIZE;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int a = a0 + u * kRotWorkers;
            if (a < n_rows) {
#pragma unroll
                for (int v = 0; v < W / 4; ++v) {
                    const uint4 g = ld_once_v4(src + (long long)a * kHeadDim * SIZE + v * 16);
                    w[u][4 * v] = g.x; w[u][4 * v + 1] = g.y; w[u][4 * v + 2] = g.z; w[u][4 * v + 3] = g.w;
                }
            }
        }
    };
    asm volatile("griddepcontrol.wait;" ::: "memory");
    load(0, worker);
    if (p.parent) {
        // how many ancestors: every node's parent in place of itself, six doublings; a warp per token
        for (int k = tid >> 5; k < here; k += kRotThreads / 32) {
            const uint32_t n = n0 + k;
            const int b = (int)(n / T), t = (int)(n % T);
            int up[2], depth[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = lane + 32 * e;
                const int par = i < p.T ? p.parent[(long long)b * p.T + i] : -1;
                up[e] = par >= 0 && par < i ? par : -1;
                depth[e] = up[e] >= 0;
            }
#pragma unroll 1
            for (int round = 0; round < 6; ++round) {
                int d2[2], u2[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int from = max(up[e], 0);
                    const int d_lo = __shfl_sync(0xffffffffu, depth[0], from & 31), d_hi = __shfl_sync(0xffffffffu, depth[1], from & 31);
                    const int u_lo = __shfl_sync(0xffffffffu, up[0], from & 31), u_hi = __shfl_sync(0xffffffffu, up[1], from & 31);
                    d2[e] = up[e] < 0 ? depth[e] : depth[e] + (from < 32 ? d_lo : d_hi);
                    u2[e] = up[e] < 0 ? -1 : from < 32 ? u_lo : u_hi;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) { depth[e] = d2[e]; up[e] = u2[e]; }
            }
            const int d_lo = __shfl_sync(0xffffffffu, depth[0], t & 31), d_hi = __shfl_sync(0xffffffffu, depth[1], t & 31);
            if (lane == 0) s_depth[k] = t < 32 ? d_lo : d_hi;
        }
        __syncthreads();
    }
    const int half = p.rot / 2;
    for (int i = tid; i < here * half; i += kRotThreads) {
        const int k = i / half, f = i % half;
        const uint32_t n = n0 + k;
        const int b = (int)(n / T), t = (int)(n % T);
        const double pos = p.positions ? (double)p.positions[n] : (double)p.seq_len[b] + (p.parent ? s_depth[k] : t);
        const double turns = pos * (p.freqs[f] * 0.15915494309189533577);            // 1 / (2 pi)
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        turn[k][f] = make_float2(c * p.factor, s * p.factor);
    }
    __syncthreads();

    for (int k = 0; k < here; ++k) {
        const uint32_t n = n0 + k;
        const int b = (int)(n / T), t = (int)(n % T);
        if (p.n_nodes && t >= p.n_nodes[b]) continue;                    // padding: left as it was
        float c[8], s[8];                                                // x cos + (the partner) s, s with the sign of its place
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = d0 + e, f = MODE == kSideBySide ? d >> 1 : d < half ? d : d - half;
            const float2 v = d < p.rot ? turn[k][f] : make_float2(1.f, 0.f);
            c[e] = v.x;
            s[e] = (MODE == kSideBySide ? e % 2 == 0 : d < half) ? -v.y : v.y;
        }
        uint8_t *const q = p.q + (long long)n * p.Hq * kRowBytes + d0 * 2, *const kv = p.kv + (long long)n * p.Hkv * 2 * kRowBytes + d0 * 2;
        const bool partly = p.rot % 8 != 0;                              // some lane holds rotated and other dims
        // the half-warps of a warp go through the rows together (rows a and a + 1)
        for (int a0 = worker; (a0 & ~1) < n_rows; a0 += kRotWorkers * AHEAD) {
            if (k > 0 || a0 > worker) load(k, a0);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int a = a0 + u * kRotWorkers;
                if ((a & ~1) >= n_rows) break;
                float x[8];
                to_floats<TYPE, W>(w[u], x);
                uint4 o = TYPE == OASIS_BF16 ? make_uint4(w[u][0], w[u][1], w[u][2], w[u][3])          // (copied bit by bit)
                                             : make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
                if ((a & ~1) < n_rot) {
                    float y[8];                                          // the partners
                    if (MODE == kSideBySide) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
                    } else if (MODE == kHalves) {
                        const int step = half >> 3, from = chunk < step ? chunk + step : chunk < 2 * step ? chunk - step : chunk;
                        uint32_t v[W];
#pragma unroll
                        for (int i = 0; i < W; ++i) v[i] = __shfl_sync(0xffffffffu, w[u][i], from, kRotLanes);
                        to_floats<TYPE, W>(v, y);
                    } else {
                        float *const row = s_row[worker];
#pragma unroll
                        for (int e = 0; e < 8; ++e) row[chunk * 9 + e] = x[e];
                        __syncwarp();
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int d = d0 + e, mate = d < half ? d + half : d < p.rot ? d - half : d;
                            y[e] = row[mate + (mate >> 3)];
                        }
                        __syncwarp();
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float r = fmaf(x[e], c[e], y[e] * s[e]);
                        x[e] = partly && d0 + e >= p.rot ? x[e] : r;
                    }
                    if (a < n_rot && d0 < p.rot)
                        o = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
                }
                if (a >= n_rows) continue;
                *reinterpret_cast<uint4 *>(a < p.Hq ? q + a * kRowBytes : kv + (a < n_rot ? 2 * (a - p.Hq) : 2 * (a - n_rot) + 1) * kRowBytes) = o;
            }
        }
    }
}

}  // namespace oasis

extern "C" int oasis_rotate_qkv(const oasis_dims_t *dims, const void *qkv, int32_t qkv_type, int64_t qkv_batch_stride, int64_t qkv_token_stride,
                                int32_t n_tokens, const int32_t *positions, const int32_t *seq_len, const int32_t *parent,
                                const int32_t *n_nodes, const double *freqs, int32_t rot_dim, int32_t interleaved, float factor, void *q,
                                void *kv, void *stream)
{
    using namespace oasis;
    const char *who = "oasis_rotate_qkv";
    if (int rc = check_dims(dims)) return rc;
    if (n_tokens < 0) return fail(OASIS_ERR_INVALID_ARG, "%s: n_tokens %d", who, n_tokens);
    if (qkv_type != OASIS_F32 && qkv_type != OASIS_BF16 && qkv_type != OASIS_F16)
        return fail(OASIS_ERR_INVALID_ARG, "%s: qkv_type %d", who, qkv_type);
    if (rot_dim < 2 || rot_dim > kHeadDim || rot_dim % 2)
        return fail(OASIS_ERR_INVALID_ARG, "%s: rot_dim %d: an even number from 2 to %d", who, rot_dim, kHeadDim);
    if (parent && (positions || !n_nodes))
        return fail(OASIS_ERR_INVALID_ARG, "%s: parent goes with n_nodes and without positions", who);
    if (parent && n_tokens > OASIS_MAX_TREE)
        return fail(OASIS_ERR_INVALID_ARG, "%s: a tree of %d nodes > %d", who, n_tokens, OASIS_MAX_TREE);
    const long long width = (long long)(dims->n_q_heads + 2ll * dims->n_kv_heads) * kHeadDim, total = (long long)dims->batch * n_tokens;
    if (n_tokens > 1 && (qkv_token_stride < width || qkv_token_stride % 8))
        return fail(OASIS_ERR_INVALID_ARG, "%s: qkv_token_stride %lld: a multiple of 8, at least %lld", who, (long long)qkv_token_stride, width);
    if (dims->batch > 1 && (qkv_batch_stride < width || qkv_batch_stride % 8))
        return fail(OASIS_ERR_INVALID_ARG, "%s: qkv_batch_stride %lld: a multiple of 8, at least %lld", who, (long long)qkv_batch_stride, width);
    if (total == 0) return OASIS_OK;
    if (!qkv || (!positions && !seq_len) || !freqs || !q || !kv) return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    if (!aligned16(qkv) || !aligned16(q) || !aligned16(kv))
        return fail(OASIS_ERR_INVALID_ARG, "%s: qkv, q and kv must be 16-byte aligned", who);
    if (total > 0x7fffffffLL) return fail(OASIS_ERR_UNSUPPORTED, "%s: more than 2^31 tokens", who);
    RotateParams p = {};
    p.qkv = (const uint8_t *)qkv; p.positions = positions; p.seq_len = seq_len; p.parent = parent; p.n_nodes = n_nodes; p.freqs = freqs;
    p.q = (uint8_t *)q; p.kv = (uint8_t *)kv; p.batch_stride = qkv_batch_stride; p.token_stride = qkv_token_stride;
    p.T = n_tokens; p.Hq = dims->n_q_heads; p.Hkv = dims->n_kv_heads; p.rot = rot_dim; p.n_tokens = total; p.factor = factor;
    // A token per thread block while that leaves SMs without work; else tokens until a half-warp has four rows to move, because
    // a thread block's start and angles have to be worth it.  Tokens per thread block: us, 65,536 tokens of 4 + 2 heads 1: 104  2: 90
    // 4: 85  8: 85; 32,768 tokens of 8 + 4 heads 1: 64  2: 59  4: 58; 8,192 of 32 + 16 heads 1: 35.9  2: 37.1  4: 38.8; 1,024 tokens
    // of 4 + 2 heads 1: 2.9  2: 3.3  4: 4.3.
    const int rows = p.Hq + 2 * p.Hkv;
    long long per = total / (8ll * sm_count());
    const long long few = (kRotWorkers * 4 + rows - 1) / rows;
    if (per > few) per = few;
    p.tokens_per_block = (int)(per < 1 ? 1 : per > kRotMaxTokens ? kRotMaxTokens : per);
    const unsigned grid = (unsigned)((total + p.tokens_per_block - 1) / p.tokens_per_block);
    const int mode = interleaved ? kSideBySide : rot_dim % 16 == 0 ? kHalves : kOddHalves;
    cudaError_t e;
#define OASIS_ROTATE(TY, MO) e = launch_waiting(rotate_qkv_kernel<TY, MO>, dim3(grid), kRotThreads, (cudaStream_t)stream, p)
#define OASIS_ROTATE_MODE(TY)                                                                                                 \
    do {                                                                                                                      \
        if (mode == kSideBySide) OASIS_ROTATE(TY, kSideBySide);                                                               \
        else if (mode == kHalves) OASIS_ROTATE(TY, kHalves);                                                                  \
        else OASIS_ROTATE(TY, kOddHalves);                                                                                    \
    } while (0)
    if (qkv_type == OASIS_F32) OASIS_ROTATE_MODE(OASIS_F32);
    else if (qkv_type == OASIS_BF16) OASIS_ROTATE_MODE(OASIS_BF16);
    else OASIS_ROTATE_MODE(OASIS_F16);
#undef OASIS_ROTATE_MODE
#undef OASIS_ROTATE
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    return OASIS_OK;
}
