// Verification of a tree of drafted tokens against the target model's logits: which path of the tree is kept, and the
// token that follows it (speculative sampling; greedy at temperature 0).
//
// The walk is serial: only after a node's distribution is known is it decided which child is next, and only the rows of
// the visited nodes are needed (2 to 5 rows of a 64-node tree).  So a request is one cluster of 1 to 8 thread blocks that
// share the vocabulary, and a visited row costs one pass and one exchange through distributed shared memory:
//   1. per node, one pass in fp32 over the row: maximum and sum of exponentials (sampling) or the first maximum (greedy).
//      The children's own logits are picked up meanwhile.
//   2. the children are tried in order, by every thread alike.  A test that the fp32 sum (off by less than kFuzzy, see
//      there) cannot decide is made with a sum in fp64: what decides is always the fp64 value.
//   3. where the walk ends, one fp64 pass gives the mass of every warp's part of the row; the part that holds the random
//      number's place in the running sum is scanned once more, in index order.  fp64, because a vocabulary of 150,000 has
//      as many borders between tokens: sums in fp32 would put a noticeable share of the draws into the neighbour's interval.
// All sums have a fixed order, so a result does not depend on timing.  The rows are re-read from L2, nothing is staged.
#include <math_constants.h>

#include "common.cuh"

namespace oasis {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerMaxCluster = 8;
// The fp32 sum of exponentials is off by less than 1e-3 of itself: a term of weight 2^-x has a relative error below
// (1.5 x + 4) 2^-23; a lane adds at most 2^22 / 512 / 4 = 2048 partial sums one after the other (2048 * 2^-24) and may
// rescale as often (2048 * 2^-22) -- 7e-4 together at the largest vocabulary.
constexpr double kFuzzy = 1e-3;

struct VerifyParams {
    const void *logits;
    const int32_t *tokens, *parent, *n_nodes;
    const float *uniforms, *temperature, *draft;
    int32_t *path, *n_commit, *next_token;
    long long lb, lr, db, dr;          // strides (elements) of logits and draft
    int T, V, M;
};

template <typename LT> struct VecOf { static constexpr int n = 16 / sizeof(LT); };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
// NaN counts as -infinity (fmaxf returns the operand that is a number).
__device__ __forceinline__ float clean(float v) { return fmaxf(v, -CUDART_INF_F); }

// One row of logits as aligned 16-byte vectors: the first `skip` elements of vector 0 belong to what lies before the row.
template <typename LT>
struct Row {
    static constexpr int N = VecOf<LT>::n;
    const LT *base;                    // 16-byte aligned; element e of vector v is row element v * N + e - skip
    int skip, V, n_vec;
    __device__ Row(const LT *row, int vocab)
    {
        skip = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(LT));
        base = row - skip;
        V = vocab;
        n_vec = (vocab + skip + N - 1) / N;
    }
    __device__ __forceinline__ int first(int v) const { return v * N - skip; }
    // The vector's logits; elements outside the row come as -infinity.
    __device__ __forceinline__ void load(int v, float (&x)[N]) const
    {
        const int i0 = first(v);
        if (i0 >= 0 && i0 + N <= V) {
            const uint4 w = *reinterpret_cast<const uint4 *>(base + (long long)v * N);
            const LT *e = reinterpret_cast<const LT *>(&w);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = clean(to_f32(e[k]));
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = (i0 + k >= 0 && i0 + k < V) ? clean(to_f32(base[(long long)v * N + k])) : -CUDART_INF_F;
        }
    }
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 bytes (two 64-bit words) to the same shared-memory place of thread block `rank` of the cluster.
__device__ __forceinline__ void st_cluster(const void *place, uint32_t rank, uint64_t a, uint64_t b)
{
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(place)), "r"(rank));
    asm volatile("st.shared::cluster.v2.u64 [%0], {%1, %2};" ::"r"(addr), "l"(a), "l"(b) : "memory");
}

struct __align__(16) Pair { uint64_t a, b; };

// What the target's distribution at the current node has become: a token's share is
//   max(a * w - b * q, 0)   with w = exp((logit - m) / temperature), tokens of `tried` left out (their q is all theirs)
struct Dist {
    float m;
    double inv_t, a, b;
    const float *q;                    // the draft's row, or NULL
    unsigned long long tried;          // rejected children (without a draft row)
};

__device__ __forceinline__ double weight(float l, const Dist &d)
{
    if (l == d.m) return 1.0;          // also where both are infinite
    return exp(((double)l - (double)d.m) * d.inv_t);
}

template <typename LT>
__global__ void __launch_bounds__(kVerThreads)
verify_tree_kernel(const VerifyParams p, const int C)
{
    constexpr int N = VecOf<LT>::n;
    __shared__ Pair s_x[2][kVerMaxCluster];            // what the thread blocks of the cluster tell one another
    __shared__ Pair s_w[kVerWarps];
    __shared__ double s_mass[kVerWarps];
    __shared__ int s_tok[OASIS_MAX_TREE], s_par[OASIS_MAX_TREE];
    __shared__ float s_u[OASIS_MAX_TREE], s_kid[OASIS_MAX_TREE], s_kq[OASIS_MAX_TREE];
    __shared__ int s_path[OASIS_MAX_TREE];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = C > 1 ? cluster_rank() : 0u;
    const int b = blockIdx.x / C;
    const int n = max(0, min(p.n_nodes[b], p.T));
    if (n == 0) {                                      // the whole cluster leaves: nothing is exchanged
        if (rank == 0) {
            for (int i = tid; i < p.M; i += kVerThreads) p.path[(long long)b * p.M + i] = -1;
            if (tid == 0) { p.n_commit[b] = 0; p.next_token[b] = -1; }
        }
        return;
    }
    for (int i = tid; i < p.T; i += kVerThreads) {
        const long long at = (long long)b * p.T + i;
        s_tok[i] = p.tokens[at];
        s_par[i] = p.parent[at];
        s_u[i] = fminf(fmaxf(p.uniforms[at], 0.f), 1.f - 5.9604645e-8f);
    }
    const float temp = p.temperature[b];
    const bool sampled = temp > 0.f;
    Dist d;
    d.inv_t = sampled ? 1.0 / (double)temp : 0.0;
    const float c2 = sampled ? fminf(1.4426950408889634f / temp, 3.0e38f) : 0.f;
    __syncthreads();
    int turn = 0;

    // A value of every thread block (two words), told to all of the cluster.  All threads of all blocks take part.
    auto exchange = [&](uint64_t x, uint64_t y) -> const Pair * {        // x, y: valid in thread 0 .. C - 1
        const Pair *got = s_x[turn];
        if (C > 1) {
            if (tid < C) st_cluster(&s_x[turn][rank], (uint32_t)tid, x, y);
            cluster_sync();
        } else {
            if (tid == 0) s_x[turn][0] = Pair{x, y};
            __syncthreads();
        }
        turn ^= 1;
        return got;
    };

    int cur = 0, n_path = 1, next = -1;
    if (tid == 0) s_path[0] = 0;
    for (;;) {
        const LT *row_ptr = reinterpret_cast<const LT *>(p.logits) + (long long)b * p.lb + (long long)cur * p.lr;
        const Row<LT> row(row_ptr, p.V);
        d.q = p.draft ? p.draft + (long long)b * p.db + (long long)cur * p.dr : nullptr;
        const int per_warp = (row.n_vec + C * kVerWarps - 1) / (C * kVerWarps);
        const int v0 = min(((int)rank * kVerWarps + warp) * per_warp, row.n_vec), v1 = min(v0 + per_warp, row.n_vec);
        // the node's children (nodes of higher index whose parent it is) and, by thread c, child c's logit
        unsigned long long kids = 0;
        if (n_path < p.M) {
            const unsigned k0 = __ballot_sync(0xffffffffu, lane > cur && lane < n && s_par[min(lane, p.T - 1)] == cur);
            const unsigned k1 = __ballot_sync(0xffffffffu, lane + 32 > cur && lane + 32 < n && s_par[min(lane + 32, p.T - 1)] == cur);
            kids = (unsigned long long)k1 << 32 | k0;
        }
        if (sampled && tid < OASIS_MAX_TREE && ((kids >> tid) & 1ull)) {
            const int t = s_tok[tid];
            const bool in = t >= 0 && t < p.V;
            s_kid[tid] = in ? clean(to_f32(row_ptr[t])) : -CUDART_INF_F;
            s_kq[tid] = in && d.q ? d.q[t] : 1.f;
        }

        if (!sampled) {
            // ---- greedy: the row's first maximum, as (value, index); equal values go to the lower index
            float best = -CUDART_INF_F;
            int at = 0x7fffffff;
            for (int v = v0 + lane; v < v1; v += 32) {
                float x[N];
                row.load(v, x);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (x[k] > best) { best = x[k]; at = row.first(v) + k; }
            }
            auto better = [](float f, int i, float g, int j) { return f > g || (f == g && i < j); };
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const float f = __shfl_xor_sync(0xffffffffu, best, o);
                const int i = __shfl_xor_sync(0xffffffffu, at, o);
                if (better(f, i, best, at)) { best = f; at = i; }
            }
            if (lane == 0) s_w[warp] = Pair{__float_as_uint(best), (uint64_t)(uint32_t)at};
            __syncthreads();
            if (tid < kVerMaxCluster) {
                for (int k = 0; k < kVerWarps; ++k) {
                    const float f = __uint_as_float((uint32_t)s_w[k].a);
                    const int i = (int)s_w[k].b;
                    if (better(f, i, best, at)) { best = f; at = i; }
                }
            }
            const Pair *got = exchange(__float_as_uint(best), (uint64_t)(uint32_t)at);
            best = -CUDART_INF_F;
            at = 0x7fffffff;
            for (int r = 0; r < C; ++r) {
                const float f = __uint_as_float((uint32_t)got[r].a);
                const int i = (int)got[r].b;
                if (better(f, i, best, at)) { best = f; at = i; }
            }
            next = best == -CUDART_INF_F ? -1 : at;
            int child = -1;
            for (unsigned long long k = kids; k && child < 0; k &= k - 1) {
                const int c = __ffsll((long long)k) - 1;
                if (next >= 0 && s_tok[c] == next) child = c;
            }
            if (child < 0) break;
            cur = child;
            if (tid == 0) s_path[n_path] = cur;
            ++n_path;
            continue;
        }

        // ---- sampled: maximum and sum of exponentials in fp32
        float m = -CUDART_INF_F, s = 0.f;
        for (int v = v0 + lane; v < v1; v += 32) {
            float x[N];
            row.load(v, x);
            float vm = x[0];
#pragma unroll
            for (int k = 1; k < N; ++k) vm = fmaxf(vm, x[k]);
            if (vm > m) {
                s *= m == -CUDART_INF_F ? 0.f : fast_exp2((m - vm) * c2);
                m = vm;
            }
            if (m == -CUDART_INF_F) continue;
            float add = 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k) add += x[k] == m ? 1.f : fast_exp2((x[k] - m) * c2);
            s += add;
        }
        auto join = [&](float &m1, float &s1, float m2, float s2) {
            const float top = fmaxf(m1, m2);
            s1 = (m1 == top ? s1 : s1 * fast_exp2((m1 - top) * c2)) + (m2 == top ? s2 : s2 * fast_exp2((m2 - top) * c2));
            m1 = top;
        };
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
            join(m, s, m2, s2);
        }
        if (lane == 0) s_w[warp] = Pair{__float_as_uint(m), __float_as_uint(s)};
        __syncthreads();
        if (tid < kVerMaxCluster) {
            m = __uint_as_float((uint32_t)s_w[0].a);
            s = __uint_as_float((uint32_t)s_w[0].b);
            for (int k = 1; k < kVerWarps; ++k) join(m, s, __uint_as_float((uint32_t)s_w[k].a), __uint_as_float((uint32_t)s_w[k].b));
        }
        const Pair *got = exchange(__float_as_uint(m), __float_as_uint(s));
        m = __uint_as_float((uint32_t)got[0].a);
        s = __uint_as_float((uint32_t)got[0].b);
        for (int r = 1; r < C; ++r) join(m, s, __uint_as_float((uint32_t)got[r].a), __uint_as_float((uint32_t)got[r].b));
        if (m == -CUDART_INF_F) break;                         // every token is left out: next stays -1
        d.m = m;
        d.a = 1.0;
        d.b = 0.0;
        d.tried = 0;

        // Mass of the row under (a, b, tried) in fp64: of every warp's part in s_mass, of the thread blocks in *parts.
        const Pair *parts = nullptr;
        auto share = [&](float x, int i, double a, double bq) -> double {      // token i's share, not normalised
            double f = weight(x, d);                           // (0 outside the row, where x is -infinity)
            if (d.q) {
                if (bq != 0.0) f = (i >= 0 && i < p.V) ? fmax(a * f - bq * (double)d.q[i], 0.0) : 0.0;
            } else {
                for (unsigned long long t = d.tried; t; t &= t - 1)
                    if (s_tok[__ffsll((long long)t) - 1] == i) f = 0.0;
            }
            return f;
        };
        auto mass = [&](double a, double bq) -> double {
            double sum = 0.0;
            for (int v = v0 + lane; v < v1; v += 32) {
                float x[N];
                row.load(v, x);
                const int i0 = row.first(v);
#pragma unroll
                for (int k = 0; k < N; ++k) sum += share(x[k], i0 + k, a, bq);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            __syncthreads();                                   // earlier readers of s_mass are done
            if (lane == 0) s_mass[warp] = sum;
            __syncthreads();
            double all = 0.0;
            if (tid < kVerMaxCluster)
                for (int k = 0; k < kVerWarps; ++k) all += s_mass[k];
            parts = exchange((uint64_t)__double_as_longlong(all), 0);
            double total = 0.0;
            for (int r = 0; r < C; ++r) total += __longlong_as_double((long long)parts[r].a);
            return total;
        };

        double z = (double)s, away = 0.0;                      // sum of all weights; weight of the tried tokens
        bool exact = false, have_mass = false;                 // z is the fp64 sum; s_mass and parts fit the distribution
        double total = 0.0;
        double ma = 1.0, mb = 0.0;                             // the (a, b) that s_mass was taken with
        int child = -1;
        for (unsigned long long k = kids; k && child < 0; k &= k - 1) {
            const int c = __ffsll((long long)k) - 1;
            const double u = (double)s_u[c];
            double w = s_kid[c] == -CUDART_INF_F ? 0.0 : weight(s_kid[c], d);
            if (d.q) {
                const double q = (double)s_kq[c];
                bool keep;
                if (d.b == 0.0) {
                    if (!exact && fabs(u * q * z - w) <= kFuzzy * (u * q * z + w)) { z = mass(1.0, 0.0); exact = true; }
                    keep = u * q < w / z;
                } else {
                    keep = u * q < fmax(d.a * w - d.b * q, 0.0);
                }
                if (keep) { child = c; break; }
                if (!exact) { z = mass(1.0, 0.0); exact = true; }
                if (d.b == 0.0) d.a = 1.0 / z;
                ma = d.a;
                mb = d.b + 1.0;
                const double rest = mass(ma, mb);
                have_mass = rest > 0.0;
                if (have_mass) {                               // (else nothing is left: p stays as it was)
                    total = rest;
                    d.a = ma / rest;
                    d.b = mb / rest;
                }
            } else {
                for (unsigned long long t = d.tried; t; t &= t - 1)
                    if (s_tok[__ffsll((long long)t) - 1] == s_tok[c]) w = 0.0;      // a sibling had the same token
                if (!exact && fabs(u * (z - away) - w) <= kFuzzy * z) { z = mass(1.0, 0.0) + away; exact = true; }
                if (u * (z - away) < w) { child = c; break; }
                away += w;
                d.tried |= 1ull << c;
            }
        }
        if (child >= 0) {
            cur = child;
            if (tid == 0) s_path[n_path] = cur;
            ++n_path;
            __syncthreads();                                   // s_kid is rewritten for the next node
            continue;
        }

        // ---- the next token: the place of uniforms[b][0] in the running sum of what is left
        if (!have_mass) {
            ma = d.a;
            mb = d.b;
            total = mass(ma, mb);
        }
        const double target = (double)s_u[0] * total;
        double before = 0.0;
        // (rounding can leave the target at the end of the last part that holds anything: then it is that part's last token)
        int owner = -1, last = 0;
        for (int r = 0; r < C && owner < 0; ++r) {
            const double part = __longlong_as_double((long long)parts[r].a);
            if (part > 0.0) last = r;
            if (target < before + part) owner = r;
            else before += part;
        }
        bool take_last = owner < 0;
        if (take_last) owner = last;
        if (owner != (int)rank) { next = -2; break; }          // another thread block writes the token
        int in_warp = -1;
        last = 0;
        for (int k = 0; k < kVerWarps && in_warp < 0; ++k) {
            if (s_mass[k] > 0.0) last = k;
            if (!take_last && target < before + s_mass[k]) in_warp = k;
            else before += s_mass[k];
        }
        take_last = take_last || in_warp < 0;
        if (in_warp < 0) in_warp = last;
        if (in_warp != warp) { next = -2; break; }             // another warp writes it
        int found = -1, last_pos = -1;
        double run_sum = before;
        for (int vb = v0; vb < v1 && found < 0; vb += 32) {
            const int v = vb + lane;
            double f[N], sum = 0.0;
            int my_last = -1;
            if (v < v1) {
                float x[N];
                row.load(v, x);
                const int i0 = row.first(v);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    f[k] = share(x[k], i0 + k, ma, mb);
                    sum += f[k];
                    if (f[k] > 0.0) my_last = i0 + k;
                }
            }
            double incl = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, !take_last && my_last >= 0 && run_sum + incl > target);
            if (hit) {
                int mine = my_last;
                if (lane == __ffs(hit) - 1) {
                    double acc = run_sum + (incl - sum);
                    const int i0 = row.first(v);
#pragma unroll
                    for (int k = N - 1; k >= 0; --k) {         // from the back: the lowest index that exceeds the target
                        double upto = acc;
#pragma unroll
                        for (int e = 0; e <= k; ++e) upto += f[e];
                        if (f[k] > 0.0 && upto > target) mine = i0 + k;
                    }
                }
                found = __shfl_sync(0xffffffffu, mine, __ffs(hit) - 1);
            }
            const unsigned any = __ballot_sync(0xffffffffu, my_last >= 0);
            if (any) last_pos = __shfl_sync(0xffffffffu, my_last, 31 - __clz(any));
            run_sum += __shfl_sync(0xffffffffu, incl, 31);
        }
        next = found >= 0 ? found : last_pos;
        break;
    }
    // greedy and empty rows: every thread knows the token, block 0 writes it; sampled: one warp does (the others have -2)
    __syncthreads();
    if (rank == 0) {
        for (int i = tid; i < p.M; i += kVerThreads) p.path[(long long)b * p.M + i] = i < n_path ? s_path[i] : -1;
        if (tid == 0) p.n_commit[b] = n_path;
    }
    if (next != -2 && lane == 0 && (next >= 0 && sampled ? true : rank == 0 && warp == 0)) p.next_token[b] = next;
}

template <typename LT>
static cudaError_t launch_verify(const VerifyParams &p, int batch, int C, cudaStream_t st)
{
    prefer_max_shared_carveout(verify_tree_kernel<LT>);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(batch * C));
    cfg.blockDim = dim3(kVerThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, verify_tree_kernel<LT>, p, C);
}

}  // namespace oasis

extern "C" int oasis_verify_tree(int32_t batch, int32_t n_tree, int32_t vocab, const void *logits, int32_t logits_type,
                                 int64_t logits_batch_stride, int64_t logits_row_stride, const int32_t *tokens,
                                 const int32_t *parent, const int32_t *n_nodes, const float *uniforms, const float *temperature,
                                 const float *draft_probs, int64_t draft_batch_stride, int64_t draft_row_stride,
                                 int32_t *path, int32_t max_path, int32_t *n_commit, int32_t *next_token, void *stream)
{
    using namespace oasis;
    const char *who = "oasis_verify_tree";
    if (batch < 0 || batch > (1 << 24)) return fail(OASIS_ERR_INVALID_ARG, "%s: batch %d", who, batch);
    if (n_tree < 1 || n_tree > OASIS_MAX_TREE)
        return fail(OASIS_ERR_INVALID_ARG, "%s: n_tree %d outside [1, %d]", who, n_tree, OASIS_MAX_TREE);
    if (vocab < 1 || vocab > OASIS_MAX_VOCAB)
        return fail(OASIS_ERR_INVALID_ARG, "%s: vocab %d outside [1, %d]", who, vocab, OASIS_MAX_VOCAB);
    if (max_path < 1 || max_path > n_tree)
        return fail(OASIS_ERR_INVALID_ARG, "%s: max_path %d outside [1, n_tree]", who, max_path);
    if (!logits || !tokens || !parent || !n_nodes || !uniforms || !temperature || !path || !n_commit || !next_token)
        return fail(OASIS_ERR_INVALID_ARG, "%s: NULL pointer argument", who);
    if (logits_type != OASIS_F32 && logits_type != OASIS_BF16 && logits_type != OASIS_F16)
        return fail(OASIS_ERR_INVALID_ARG, "%s: logits_type %d", who, logits_type);
    const uintptr_t size = logits_type == OASIS_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(draft_probs) % 4)
        return fail(OASIS_ERR_INVALID_ARG, "%s: logits and draft_probs must be aligned to their type", who);
    if (logits_row_stride < vocab || logits_batch_stride < 0 || (draft_probs && (draft_row_stride < vocab || draft_batch_stride < 0)))
        return fail(OASIS_ERR_INVALID_ARG, "%s: row strides %lld, %lld of %d logits", who, (long long)logits_row_stride,
                    (long long)draft_row_stride, vocab);
    if (batch == 0) return OASIS_OK;
    VerifyParams p;
    p.logits = logits; p.tokens = tokens; p.parent = parent; p.n_nodes = n_nodes; p.uniforms = uniforms;
    p.temperature = temperature; p.draft = draft_probs; p.path = path; p.n_commit = n_commit; p.next_token = next_token;
    p.lb = logits_batch_stride; p.lr = logits_row_stride; p.db = draft_batch_stride; p.dr = draft_row_stride;
    p.T = n_tree; p.V = vocab; p.M = max_path;
    // as many thread blocks per request as the SMs take at two each, at least 2,048 tokens for each
    int C = kVerMaxCluster;
    while (C > 1 && ((long long)batch * C > 2ll * sm_count() || vocab < C * 2048)) C >>= 1;
    cudaError_t e;
    if (logits_type == OASIS_F32) e = launch_verify<float>(p, batch, C, (cudaStream_t)stream);
    else if (logits_type == OASIS_BF16) e = launch_verify<__nv_bfloat16>(p, batch, C, (cudaStream_t)stream);
    else e = launch_verify<__half>(p, batch, C, (cudaStream_t)stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    return check_launch(who);
}
