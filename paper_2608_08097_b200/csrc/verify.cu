// Verification of a tree of drafted tokens against the target model's logits: which path of the tree is kept, and the
// token that follows it (speculative sampling; greedy at temperature 0).
//
// The walk is serial: only after a node's distribution is known is it decided which child is next, and only the rows of
// the visited nodes are needed (2 to 5 rows of a 64-node tree).  So a request is one cluster of 1 to 8 thread blocks that
// share the vocabulary, and a visited row costs one pass and one exchange:
//   1. per node, every warp copies its part of the row into shared memory (cp.async) and makes one pass in fp32 over it:
//      maximum and sum of exponentials (sampling) or the first maximum (greedy).  The warps' results go to every block of
//      the cluster by asynchronous stores into shared memory, which an mbarrier counts.
//   2. warp 0 of each block then tries the children in order, all blocks alike, while the other warps wait: serial code
//      that every warp ran would take the issue slots of the one that matters.  A test that the fp32 sum (off by less than
//      kFuzzy, see there) cannot decide is made with a sum in fp64: what decides is always the fp64 value.
//   3. where the walk ends, one fp64 pass over the staged part gives every warp's mass; the part that holds the random
//      number's place in the running sum is scanned once more, in index order.  fp64, because a vocabulary of 150,000 has
//      as many borders between tokens: sums in fp32 would put a noticeable share of the draws into the neighbour's interval.
// All sums have a fixed order, so a result does not depend on timing.
// What bounds it: the latency of the serial steps, not bytes.  16 requests, 64-node trees, 151,936 bf16 logits: 28.1 us, of
// which (cycles) start 4,500, each node 9,000 (copy 2,000, fp32 pass 2,900, exchange 1,300, decision 2,700), the fp64 pass
// 9,800, the search 1,700.  One request, greedy, 32,000 logits: 7.7 us.  16 requests, chains of 5 with draft distributions,
// 128,256 fp32 logits: 40.4 us.  128 requests, 6 nodes, 50,257 fp16 logits: 30.6 us.  (In a graph.  The launch may overlap the
// end of the previous kernel, which it waits for before it reads any input: that saves 1.5 to 2.4 us a call where calls are
// launched one by one.)  No launch_dependents here: it gains 0.5 to 1 us for one request and for 128 and costs the chains 3 us,
// whose successors' thread blocks then take the places beside theirs.
#include <math_constants.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace oasis {

constexpr int kVerMaxCluster = 8;
// The fp32 sum of exponentials is off by less than 3e-4 of itself, and 2e-3 is taken for it:
//   m c2, below 4096, is rounded once per lane and chunk (2^-12 in the exponent)                                1.7e-4
//   a term of weight 2^-x has a relative error below (1.5 x + 4) 2^-23; x is below 20 on the weighted average     4e-6
//   a lane adds the terms of a chunk, 17 vectors at most (blocks of 512 threads; 16 with 256), to two accumulators
//   (34 additions each; the careful loop 136 to one)                                                             8e-6
//   then chunk after chunk, each a rescaling by an exponential (2^-22) and an addition: 257 chunks at most
//   (2^22 fp32 logits, one block of 256 threads)                                                                8e-5
//   and twelve such steps over the lanes, warps and thread blocks                                                4e-6
constexpr double kFuzzy = 2e-3;
// A weight reaches down to e^-600 = 1e-260: it, its share after a rejection that left only such tokens (times 1e260) and what
// further rejections cancel of that stay within the range of a double.
constexpr float kReach = 600.f;

struct VerifyParams {
    const void *logits;
    const int32_t *tokens, *parent, *n_nodes;
    const float *uniforms, *temperature, *draft;
    int32_t *path, *n_commit, *next_token, *err;
    long long lb, lr, db, dr;          // strides (elements) of logits and draft
    int T, V, M;
};

template <typename LT> struct Logit;                   // elements per 16-byte vector, the pattern of -infinity, unpacking
template <> struct Logit<float> {
    static constexpr int N = 4;
    static constexpr uint32_t kNone = 0xff800000u;
    static __device__ __forceinline__ float get(const uint4 &w, int k) { return __uint_as_float((&w.x)[k]); }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
};
template <> struct Logit<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t kNone = 0xff80u;
    static __device__ __forceinline__ float get(const uint4 &w, int k)
    {
        const uint32_t h = (&w.x)[k >> 1];
        return __uint_as_float((k & 1) ? (h & 0xffff0000u) : (h << 16));
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
};
template <> struct Logit<__half> {
    static constexpr int N = 8;
    static constexpr uint32_t kNone = 0xfc00u;
    static __device__ __forceinline__ float get(const uint4 &w, int k)
    {
        const uint32_t h = (&w.x)[k >> 1];
        return __half2float(__ushort_as_half((unsigned short)((k & 1) ? (h >> 16) : (h & 0xffffu))));
    }
    static __device__ __forceinline__ float one(const __half *p) { return __half2float(*p); }
};
// NaN counts as -infinity (fmaxf returns the operand that is a number).
__device__ __forceinline__ float clean(float v) { return fmaxf(v, -CUDART_INF_F); }

// Sets element k of a vector in shared memory to -infinity.
template <typename LT>
__device__ __forceinline__ void leave_out(uint4 *w, int k)
{
    if (sizeof(LT) == 4) reinterpret_cast<uint32_t *>(w)[k] = Logit<LT>::kNone;
    else reinterpret_cast<uint16_t *>(w)[k] = (uint16_t)Logit<LT>::kNone;
}

// One row of logits as aligned 16-byte vectors: the first `skip` elements of vector 0 belong to what lies before the row.
template <typename LT>
struct Row {
    static constexpr int N = Logit<LT>::N;
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
    // This lane's vectors v, v + 32, ... below v_end to dst, dst + 32, ... by asynchronous copies (complete after
    // stage_wait); what lies outside the row comes as -infinity.
    __device__ __forceinline__ void stage(int v, int v_end, uint4 *dst) const
    {
        const int lo = skip ? 1 : 0, hi = (V + skip) / N;              // the vectors that lie inside the row
        const LT *src = base + (long long)v * N;
#pragma unroll 4
        for (int i = v; i < v_end; i += 32, src += 32 * N)
            if (i >= lo && i < hi)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst + (i - v))), "l"(src) : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (skip && v == 0 && v_end > 0) edge(base, -skip, V, dst);
        if (hi < n_vec && hi >= lo && hi >= v && hi < v_end && ((hi - v) & 31) == 0) edge(base + (long long)hi * N, hi * N - skip, V, dst + (hi - v));
    }
    // The row's first or last vector, whose element 0 is row element i0.
    static __device__ __noinline__ void edge(const LT *src, int i0, int V, uint4 *dst)
    {
        for (int k = 0; k < N; ++k) {
            if (i0 + k >= 0 && i0 + k < V) reinterpret_cast<LT *>(dst)[k] = src[k];
            else leave_out<LT>(dst, k);
        }
    }
};
__device__ __forceinline__ void stage_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

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
// 16 bytes (two 64-bit words) to the same shared-memory place of thread block `rank` of the cluster, counted by its mbarrier.
__device__ __forceinline__ void send(const void *place, uint32_t bar, uint32_t rank, uint64_t a, uint64_t b)
{
    uint32_t addr, rbar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(place)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rbar) : "r"(bar), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(addr), "l"(a), "l"(b), "r"(rbar)
                 : "memory");
}

struct __align__(16) Pair { uint64_t a, b; };

// The target's distribution at the current node: a token's weight is w = exp((logit - m) / temperature).  Rejected tokens leave
// the row; under a draft row q, k rejections leave a token with r_k, where r_0 = w and r_j = max(s_{j-1} r_{j-1} - q, 0), s_j being one
// over the sum of all r_j, and with the share s_k r_k.  (Folded into one product a w - b q, what is 0 after one rejection came
// back out of the rounding of large a and b after the next.)
struct Dist {
    float l_min;                       // logits up to here have weight 0: kReach temperatures below m, and everything but m at tiny ones
    double m, c;                       // c = 64 log2(e) / temperature
    const float *q;                    // the draft's row, or NULL
    int k;                             // rejections against it so far
};

// 2^(j / 64), made at compile time from square roots (Newton's iteration) of two: the binary digits of j pick the factors.
// Sixteen copies of each, so that the 16 lanes of a shared-memory wavefront read 16 different banks whatever their j.
constexpr int kExpSteps = 64, kExpCopies = 16, kExpTable = kExpSteps * kExpCopies;
struct ExpTable {
    double v[kExpTable];
    constexpr ExpTable() : v()
    {
        double root[6] = {};
        double x = 2.0;
        for (int i = 5; i >= 0; --i) {                     // root[i] = 2^(2^i / 64)
            double y = 1.0 + (x - 1.0) / 2;
            for (int k = 0; k < 8; ++k) y = (y + x / y) / 2;
            x = root[i] = y;
        }
        for (int j = 0; j < kExpSteps; ++j) {
            double f = 1.0;
            for (int i = 0; i < 6; ++i)
                if ((j >> i) & 1) f *= root[i];
            for (int k = 0; k < kExpCopies; ++k) v[j * kExpCopies + k] = f;
        }
    }
};
__device__ const ExpTable g_exp_table = ExpTable();

// exp((l - m) / temperature) in fp64, to about 1e-13 of itself.  With y = (l - m) c and n = y rounded to a whole number,
//   2^(y / 64) = 2^floor(n / 64) * T[n mod 64] * exp(z),  z = (y - n) ln 2 / 64,  |z| <= 0.0055,
// and four terms of the series for exp(z) - 1 leave 4e-14; y's own rounding adds up to 1.3e-13 at the smallest weights.  All bits are
// kept: where a draft row nearly agrees with the target their difference is a 2^-25 or less of either, and cut to 33 bits (which
// this was once, for sums of equal weights to be exact) it chose another token in 2 of 512 draws.  This is the pass over
// 152,000 logits that the last node of every walk needs; exp() takes 2.5 times as long (19.7 against 7.8 cycles per 32
// logits and SM, with a table of 1,024 steps that had bank conflicts).
__device__ __forceinline__ double weight(float l, const Dist &d, const double *table)       // table: this lane's copy
{
    constexpr double kStep = 0.69314718055994530942 / kExpSteps, kRound = 6755399441055744.0;   // 1.5 * 2^52
    const double y = ((double)l - d.m) * d.c;
    const double t = y + kRound;
    const int n = __double2loint(t);
    const double r = y - (t - kRound);
    const double f = table[(n & (kExpSteps - 1)) * kExpCopies];
    const double e = fma(r, fma(r, fma(r, kStep * kStep * kStep * kStep / 24, kStep * kStep * kStep / 6), kStep * kStep / 2), kStep);
    const double w = fma(f * r, e, f);
    const double scaled = __hiloint2double(__double2hiint(w) + ((n & ~(kExpSteps - 1)) << 14), __double2loint(w));
    return l > d.l_min ? scaled : 0.0;                     // (also for NaN and -infinity)
}

__device__ __forceinline__ double shfl_d(double v, int lane) { return __shfl_sync(0xffffffffu, v, lane); }

// What warp 0 decides and the other warps carry out.
enum { kGo = 0, kMass = 1, kSearch = 2, kEnd = 3 };        // on to a child | a mass pass | find the next token | done
struct Control {
    int cmd, cur, ahead;               // ahead: the likeliest node after cur, or -1
    int infinite;                      // some logit of the row is +infinity
    unsigned long long tried;          // rejected children (without a draft row)
    Dist d;
    double s[OASIS_MAX_TREE];          // s_0 .. s_k
    int pass;                          // the mass pass sums r_pass
    // kept by warp 0 from one decision about a node to the next
    double z, away;                    // sum of the weights when it was last measured; weight of the tokens tried since
    unsigned long long left;           // children not tried yet
    int exact, have_mass, need;        // z is the fp64 sum; s_mass fits the distribution; what the mass pass is for
    // the search
    double target, before;
    int in_warp, take_last;            // (in_warp -1: another thread block has it)
};

// r_k, k > 0, of a token with weight w and draft share q.
__device__ __forceinline__ double left_of(double w, double q, int k, double s0, const Control &ctl)
{
    double r = fmax(s0 * w - q, 0.0);
#pragma unroll 1
    for (int j = 1; j < k; ++j) r = fmax(ctl.s[j] * r - q, 0.0);
    return r;
}

// One chunk of a warp's vectors: the sum of r_pass of every vector goes to my_sum, the lane's sum is returned.  Tokens
// that were tried leave the row by turning their logits into -infinity.
template <typename LT>
__device__ __noinline__ double chunk_mass(const Control &ctl, const Row<LT> &row, int vc, int ve, int lane, bool reload, uint4 *my_row,
                                          double *my_sum, const double *table, const int *s_tok)
{
    constexpr int N = Logit<LT>::N;
    if (reload) { row.stage(vc + lane, ve, my_row); stage_wait(); }
#pragma unroll 1
    for (unsigned long long t = ctl.tried; t; t &= t - 1) {
        const int token = s_tok[__ffsll((long long)t) - 1], e = token + row.skip, v = e / N;
        if (token >= 0 && token < row.V && v >= vc && v < ve && ((v - vc) & 31) == lane) leave_out<LT>(my_row + (v - vc - lane), e % N);
    }
    const Dist d = ctl.d;
    const int pass = ctl.pass;
    const double s0 = ctl.s[0];
    const double *const my_table = table + (lane & (kExpCopies - 1));
    double sum = 0.0;
    if (d.q && pass == 0)                                          // a pass under the draft's row may follow: on its way to L2
        for (int i = max(row.first(vc), 0) + lane * 32; i < min(row.first(ve), row.V); i += 32 * 32)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(d.q + i));
    if (pass == 0 && !ctl.infinite) {
#pragma unroll 1
        for (int v = vc + lane; v < ve; v += 32) {
            const uint4 w = my_row[v - vc - lane];
            double f[N];
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = weight(Logit<LT>::get(w, k), d, my_table);
#pragma unroll
            for (int o = 1; o < N; o <<= 1)
#pragma unroll
                for (int k = 0; k < N; k += 2 * o) f[k] += f[k + o];
            const double part = f[0];
            my_sum[v - vc - lane] = part;
            sum += part;
        }
    } else {
        float q[N], q_next[N];
        auto fetch = [&](int v, float (&f)[N]) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = row.first(v) + k;
                f[k] = pass > 0 && v < ve && i >= 0 && i < row.V ? d.q[i] : 0.f;
            }
        };
        const bool plain = !ctl.infinite && pass == 1;              // (the others are rare)
        fetch(vc + lane, q);
#pragma unroll 1
        for (int v = vc + lane; v < ve; v += 32) {
            fetch(v + 32, q_next);
            const uint4 w = my_row[v - vc - lane];
            double part = 0.0;
            if (plain) {
#pragma unroll
                for (int k = 0; k < N; ++k)                        // (outside the row the logit is -infinity)
                    part += fmax(s0 * weight(Logit<LT>::get(w, k), d, my_table) - (double)q[k], 0.0);
            } else {
#pragma unroll 1
                for (int k = 0; k < N; ++k) {
                    const float l = Logit<LT>::one(reinterpret_cast<const LT *>(my_row + (v - vc - lane)) + k);
                    const double f = weight(!ctl.infinite ? l : l == CUDART_INF_F ? 0.f : -CUDART_INF_F, d, my_table);
                    const int i = row.first(v) + k;
                    part += pass == 0 ? f : i >= 0 && i < row.V ? left_of(f, (double)d.q[i], pass, s0, ctl) : 0.0;
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k) q[k] = q_next[k];
            my_sum[v - vc - lane] = part;
            sum += part;
        }
    }
    return sum;
}

// cap: vectors per warp that shared memory holds.  A part of the row that is not larger (n_chunks == 1) is read once per
// visited node, whatever happens there; a larger one is read again for every pass.
// Between the passes warp 0 alone talks to the other thread blocks of the cluster and decides; that every warp did it cost
// more than the passes (four warps per scheduler running the same 200 serial instructions).
template <typename LT, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
verify_tree_kernel(const VerifyParams p, const int C, const int cap)
{
    constexpr int N = Logit<LT>::N, WARPS = THREADS / 32;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ Pair s_x[2][kVerMaxCluster];            // what the thread blocks of the cluster tell one another
    __shared__ __align__(8) uint64_t s_bar[2];
    __shared__ Pair s_w[WARPS];
    __shared__ double s_mass[WARPS];
    __shared__ __align__(16) double s_table[kExpTable];
    __shared__ int s_tok[OASIS_MAX_TREE], s_par[OASIS_MAX_TREE];
    __shared__ float s_u[OASIS_MAX_TREE];
    __shared__ int s_path[OASIS_MAX_TREE];
    __shared__ Control ctl;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint4 *const my_row = reinterpret_cast<uint4 *>(smem_raw) + warp * cap + lane;              // this lane's vectors, 32 apart
    double *const my_sum = reinterpret_cast<double *>(smem_raw + (size_t)WARPS * cap * 16) + warp * cap + lane;   // their masses
    const uint32_t rank = C > 1 ? cluster_rank() : 0u;
    const int b = blockIdx.x / C;
    const LT *const logits = reinterpret_cast<const LT *>(p.logits) + (long long)b * p.lb;
    const int parts_of_row = C * WARPS, part = (int)rank * WARPS + warp;
    // this warp's vectors of node x's row, and their way into shared memory
    Row<LT> row(logits, p.V);
    int v0 = 0, v1 = 0, n_chunks = 1;
    auto enter = [&](int x) {
        row = Row<LT>(logits + (long long)x * p.lr, p.V);
        const int per_warp = (row.n_vec + parts_of_row - 1) / parts_of_row;
        v0 = min(part * per_warp, row.n_vec);
        v1 = min(v0 + per_warp, row.n_vec);
        n_chunks = (per_warp + cap - 1) / cap;         // the same for all warps
        row.stage(v0 + lane, min(v0 + cap, v1), my_row);
    };
    // What needs no input may run before the previous kernel in the stream has ended: the table of the weights, the barriers
    // (the cluster's own barrier comes later, beside the first row's copy: in front of it it would cost the chains 2.2 us).
    for (int i = 2 * tid; i < kExpTable; i += 2 * THREADS)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(s_table + i)), "l"(g_exp_table.v + i) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (tid == 0) {
        mbar_init(smem_u32(&s_bar[0]), 1);
        mbar_init(smem_u32(&s_bar[1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    enter(0);                                          // node 0's row is needed in any case
    const int n = max(0, min(p.n_nodes[b], p.T));
    const float temp = p.temperature[b];
    int tok = 0, par = -1;
    float un = 0.f;
    if (tid < p.T) {
        const long long at = (long long)b * p.T + tid;
        tok = p.tokens[at];
        par = p.parent[at];
        un = p.uniforms[at];
    }
    if (n == 0) {                                      // the whole cluster leaves: nothing is exchanged
        stage_wait();
        if (rank == 0) {
            for (int i = tid; i < p.M; i += THREADS) p.path[(long long)b * p.M + i] = -1;
            if (tid == 0) { p.n_commit[b] = 0; p.next_token[b] = -1; }
        }
        return;
    }
    const bool sampled = temp > 0.f;
    if (tid < OASIS_MAX_TREE) {
        s_tok[tid] = tok;
        s_par[tid] = par;
        s_u[tid] = fminf(fmaxf(un, 0.f), 1.f - 5.9604645e-8f);
    }
    // (kept away from 0 and infinity: a logit of -infinity has weight 0 at any temperature)
    const float c2 = fmaxf(fminf(1.4426950408889634f / temp, 3.0e38f), 1.2e-38f);
    if (tid == 0) {
        s_path[0] = 0;
        ctl.ahead = n > 1 ? 1 : -1;
        ctl.d.c = kExpSteps * 1.4426950408889634 * (sampled ? fmax(1.0 / (double)temp, 1e-300) : 0.0);
    }
    if (C > 1) cluster_sync();                         // the barriers of all blocks are there
    else __syncthreads();

    int turn = 0;                                      // exchanges so far
    int n_path = 1, next = -1;
    for (;;) {
        const int cur = n_path == 1 ? 0 : ctl.cur;
        const LT *const row_ptr = logits + (long long)cur * p.lr;
        const float *const q_row = p.draft ? p.draft + (long long)b * p.db + (long long)cur * p.dr : nullptr;
        const int ahead = ctl.ahead;
        if (ahead >= 0) {                              // the likeliest next row on its way to L2
            const Row<LT> next_row(logits + (long long)ahead * p.lr, p.V);
            for (int v = v0 + lane * 8; v < min(v1, next_row.n_vec); v += 32 * 8)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(next_row.base + (long long)v * N));
        }
        // warp 0: the node's children (nodes of higher index whose parent it is); lane c holds the logits of children c, c + 32
        unsigned kids0 = 0, kids1 = 0;
        float kid0 = -CUDART_INF_F, kid1 = -CUDART_INF_F, kq0 = 1.f, kq1 = 1.f;
        if (warp == 0 && n_path < p.M) {
            kids0 = __ballot_sync(0xffffffffu, lane > cur && lane < n && s_par[lane] == cur);
            kids1 = __ballot_sync(0xffffffffu, lane + 32 > cur && lane + 32 < n && s_par[lane + 32] == cur);
            if (sampled && ((kids0 >> lane) & 1u) && (unsigned)s_tok[lane] < (unsigned)p.V) {
                kid0 = Logit<LT>::one(row_ptr + s_tok[lane]);
                if (q_row) kq0 = q_row[s_tok[lane]];
            }
            if (sampled && ((kids1 >> lane) & 1u) && (unsigned)s_tok[lane + 32] < (unsigned)p.V) {
                kid1 = Logit<LT>::one(row_ptr + s_tok[lane + 32]);
                if (q_row) kq1 = q_row[s_tok[lane + 32]];
            }
        }
        stage_wait();

        // ---- one pass over the row
        if (!sampled) {
            // greedy: the first maximum, as one key: value (order-preserving, -0 as +0), then the lower index
            unsigned long long best = 0;
            for (int ch = 0; ch < n_chunks; ++ch) {
                const int vc = v0 + cap * ch, ve = min(vc + cap, v1);
                if (ch > 0) { row.stage(vc + lane, ve, my_row); stage_wait(); }
                float top = -CUDART_INF_F;
                int at = 0;
#pragma unroll 2
                for (int v = vc + lane; v < ve; v += 32) {
                    const uint4 w = my_row[v - vc - lane];
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const float x = Logit<LT>::get(w, k);                    // (a NaN is not larger)
                        if (x > top) { top = x; at = row.first(v) + k; }
                    }
                }
                const uint32_t u = __float_as_uint(top + 0.f), key = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
                const unsigned long long full = (unsigned long long)key << 32 | (0xffffffffu - (uint32_t)at);
                if (top > -CUDART_INF_F && full > best) best = full;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
            if (lane == 0) s_w[warp].a = best;
        } else {
            // sampled: maximum and sum of exponentials in fp32
            float m = -CUDART_INF_F, s = 0.f;
            for (int ch = 0; ch < n_chunks; ++ch) {
                const int vc = v0 + cap * ch, ve = min(vc + cap, v1);
                if (ch > 0) { row.stage(vc + lane, ve, my_row); stage_wait(); }
                float top = -CUDART_INF_F;
#pragma unroll 4
                for (int v = vc + lane; v < ve; v += 32) {
                    const uint4 w = my_row[v - vc - lane];
#pragma unroll
                    for (int k = 0; k < N; k += 2) top = max3(top, Logit<LT>::get(w, k), Logit<LT>::get(w, k + 1));   // (a NaN loses)
                }
                if (top > m) {
                    s *= m == -CUDART_INF_F ? 0.f : fast_exp2((m - top) * c2);
                    m = top;
                }
                if (m == -CUDART_INF_F) continue;
                // x c2 - m c2 as one packed multiply-add for two logits; the rounding of m c2 is a common factor, off by less
                // than 2^-12 as long as |m c2| < 4096.  Rows with larger ones, NaN or infinities take the careful loop.
                const float mc = -m * c2;
                float sum = CUDART_INF_F;
                if (fabsf(mc) < 4096.f) {
                    const uint64_t c22 = f32x2(c2, c2), mc2 = f32x2(mc, mc);
                    uint64_t acc[2] = {0ull, 0ull};
#pragma unroll 4
                    for (int v = vc + lane; v < ve; v += 32) {
                        const uint4 w = my_row[v - vc - lane];
#pragma unroll
                        for (int k = 0; k < N; k += 2) {
                            float e0, e1;
                            f32x2_split(fma_f32x2(f32x2(Logit<LT>::get(w, k), Logit<LT>::get(w, k + 1)), c22, mc2), e0, e1);
                            acc[(k >> 1) & 1] = add_f32x2(acc[(k >> 1) & 1], f32x2(fast_exp2(e0), fast_exp2(e1)));
                        }
                    }
                    float a0, a1;
                    f32x2_split(add_f32x2(acc[0], acc[1]), a0, a1);
                    sum = a0 + a1;
                }
                if (!(sum < 1e30f)) {
                    sum = 0.f;
#pragma unroll 1
                    for (int v = vc + lane; v < ve; v += 32) {
                        const uint4 w = my_row[v - vc - lane];
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            const float x = clean(Logit<LT>::get(w, k));
                            sum += x == m ? 1.f : fast_exp2((x - m) * c2);
                        }
                    }
                }
                s += sum;
            }
            float top = m;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            s = m == top ? s : s * fast_exp2((m - top) * c2);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0) s_w[warp] = Pair{__float_as_uint(top), __float_as_uint(s)};
        }
        __syncthreads();

        // ---- decisions (warp 0), and mass passes between them
        for (bool first = true;; first = false) {
            if (warp == 0) {
                // the block's value, then the cluster's
                uint64_t x0, x1 = 0;
                float m = 0.f, s = 0.f;
                if (!first) {
                    double all = s_mass[lane & (WARPS - 1)];
#pragma unroll
                    for (int o = WARPS / 2; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
                    x0 = (uint64_t)__double_as_longlong(all);
                } else {
                    const Pair mine = s_w[lane & (WARPS - 1)];
                    x0 = mine.a;
                    if (!sampled) {
#pragma unroll
                        for (int o = WARPS / 2; o > 0; o >>= 1) x0 = max((unsigned long long)x0, __shfl_xor_sync(0xffffffffu, (unsigned long long)x0, o));
                    } else {
                        m = __uint_as_float((uint32_t)mine.a);
                        s = __uint_as_float((uint32_t)mine.b);
                        float top = m;
#pragma unroll
                        for (int o = WARPS / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        s = m == top ? s : s * fast_exp2((m - top) * c2);
#pragma unroll
                        for (int o = WARPS / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                        x0 = __float_as_uint(top);
                        x1 = __float_as_uint(s);
                    }
                }
                const Pair *got = s_x[turn & 1];
                bool alive = true;
                if (C > 1) {
                    const uint32_t bar = smem_u32(&s_bar[turn & 1]);
                    if (lane < C) send(&s_x[turn & 1][rank], bar, (uint32_t)lane, x0, x1);
                    if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)C * 16u);
                    __syncwarp();
                    // (two lanes probe in a predicated instruction: a wait inside `if (lane == 0)` left the warp diverged)
                    alive = mbar_wait_warp2(bar, (uint32_t)(turn >> 1) & 1u, bar, (uint32_t)(turn >> 1) & 1u, p.err, 81);
                } else {
                    if (lane == 0) s_x[turn & 1][0] = Pair{x0, x1};
                    __syncwarp();
                }
                ++turn;
                const bool from = lane < C;                       // lane r holds what block r told, the others nothing
                const Pair theirs = got[from ? lane : 0];
                int cmd = kMass, child = -1;
                if (!alive) {
                    cmd = kEnd;
                } else if (!sampled) {
                    unsigned long long best = from ? theirs.a : 0;
#pragma unroll
                    for (int o = kVerMaxCluster / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
                    best = __shfl_sync(0xffffffffu, best, 0);
                    next = best == 0 ? -1 : (int)(0xffffffffu - (uint32_t)best);  // 0: every token is left out
                    const unsigned e0 = __ballot_sync(0xffffffffu, ((kids0 >> lane) & 1u) && s_tok[lane] == next);
                    const unsigned e1 = __ballot_sync(0xffffffffu, ((kids1 >> lane) & 1u) && s_tok[lane + 32] == next);
                    if (next >= 0) child = e0 ? __ffs(e0) - 1 : e1 ? __ffs(e1) + 31 : -1;
                    cmd = child >= 0 ? kGo : kEnd;
                } else {
                    Dist d = ctl.d;
                    double z = ctl.z, away = ctl.away, total = 0.0;
                    unsigned long long left = ctl.left, tried = ctl.tried;
                    bool exact = ctl.exact, have_mass = ctl.have_mass;
                    int need = ctl.need;
                    enum { kNothing, kExact, kRest, kFinal };
                    if (first) {
                        m = from ? __uint_as_float((uint32_t)theirs.a) : -CUDART_INF_F;
                        s = from ? __uint_as_float((uint32_t)theirs.b) : 0.f;
                        float top = m;
#pragma unroll
                        for (int o = kVerMaxCluster / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        s = m == top ? s : s * fast_exp2((m - top) * c2);
#pragma unroll
                        for (int o = kVerMaxCluster / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                        top = __shfl_sync(0xffffffffu, top, 0);
                        s = __shfl_sync(0xffffffffu, s, 0);
                        // tokens with a logit of +infinity share everything: such a row reads as 0 at them and -infinity elsewhere
                        const bool infinite = top == CUDART_INF_F;
                        if (infinite) {
                            kid0 = kid0 == CUDART_INF_F ? 0.f : -CUDART_INF_F;
                            kid1 = kid1 == CUDART_INF_F ? 0.f : -CUDART_INF_F;
                        }
                        const float at = infinite ? 0.f : top;
                        d.m = (double)at;
                        d.l_min = fminf(at - kReach * temp, nextafterf(at, -CUDART_INF_F));
                        d.q = q_row;
                        d.k = 0;
                        z = (double)s;
                        away = 0.0;
                        left = (unsigned long long)kids1 << 32 | kids0;
                        tried = 0;
                        exact = have_mass = false;
                        if (lane == 0) ctl.infinite = infinite;
                        if (top == -CUDART_INF_F) { cmd = kEnd; left = 0; }          // every token is left out: next stays -1
                    } else {
                        double mass = 0.0;
                        for (int r = 0; r < C; ++r) mass += __longlong_as_double((long long)got[r].a);
                        if (need == kExact) {                                       // of what is left: tried tokens have left the row
                            z = mass;
                            away = 0.0;
                            exact = true;
                        } else {
                            have_mass = need == kFinal || mass > 0.0;               // (else nothing is left: p stays as it was)
                            if (have_mass) total = mass;
                            if (need == kRest && have_mass) {
                                d.k = ctl.pass;
                                if (lane == 0) ctl.s[d.k] = 1.0 / mass;
                                __syncwarp();
                            }
                        }
                        if (have_mass && need == kExact) have_mass = false;         // (s_mass was used for something else)
                    }
                    // The children in order.  Whatever needs the row's mass in fp64 (a close decision, a rejection against
                    // a draft row, the next token) asks for a pass and comes back.
                    const double w0 = weight(kid0, d, s_table + (lane & (kExpCopies - 1)));
                    const double w1 = left >> 32 ? weight(kid1, d, s_table + (lane & (kExpCopies - 1))) : 0.0;
                    need = kNothing;
#pragma unroll 1
                    while (left) {
                        const int i = __ffsll((long long)left) - 1;
                        const double u = (double)s_u[i];
                        double wc = shfl_d(i < 32 ? w0 : w1, i & 31);
                        if (q_row) {
                            const double q = (double)__shfl_sync(0xffffffffu, i < 32 ? kq0 : kq1, i & 31);
                            const double uq = u * q;
                            if (d.k == 0 && !exact && fabs(uq * z - wc) <= kFuzzy * (uq * z + wc)) { need = kExact; break; }
                            const double share = d.k == 0 ? wc / z : ctl.s[d.k] * left_of(wc, q, d.k, ctl.s[0], ctl);
                            if (uq < share) { child = i; break; }
                            if (!exact) { need = kExact; break; }
                            if (d.k == 0 && lane == 0) ctl.s[0] = 1.0 / z;
                            left &= left - 1;
                            need = kRest;
                            break;
                        }
                        for (unsigned long long t = tried; t; t &= t - 1)
                            if (s_tok[__ffsll((long long)t) - 1] == s_tok[i]) wc = 0.0;          // a sibling had the same token
                        if (!exact && fabs(u * (z - away) - wc) <= kFuzzy * z) { need = kExact; break; }
                        if (u * (z - away) < wc) { child = i; break; }
                        away += wc;
                        // Where a rejection leaves less than 2^-10 of the measured sum, z - away has lost more than ten of its bits:
                        // what is left is measured again (random numbers close to 1; four tokens in a row of 2^-24 each lost them all).
                        if (z - away < 0x1p-10 * z) exact = false;
                        tried |= 1ull << i;
                        left &= left - 1;
                    }
                    if (child >= 0) {
                        cmd = kGo;
                    } else if (cmd != kEnd && need == kNothing && have_mass) {
                        // the next token: the place of uniforms[b][0] in the running sum of what is left.  (Rounding can leave
                        // the target at the end of the last part that holds anything: then it is that part's last token.)
                        cmd = kSearch;
                        const double target = (double)s_u[0] * total;
                        double before = 0.0;
                        int owner = -1, last = 0;
                        for (int r = 0; r < C && owner < 0; ++r) {
                            const double mine = __longlong_as_double((long long)got[r].a);
                            if (mine > 0.0) last = r;
                            if (target < before + mine) owner = r;
                            else before += mine;
                        }
                        const bool take_last = owner < 0;
                        if (take_last) owner = last;
                        int in_warp = -1;
                        if (owner == (int)rank) {
                            last = 0;
                            for (int k = 0; k < WARPS && in_warp < 0; ++k) {
                                if (s_mass[k] > 0.0) last = k;
                                if (!take_last && target < before + s_mass[k]) in_warp = k;
                                else before += s_mass[k];
                            }
                        }
                        if (lane == 0) {
                            ctl.target = target;
                            ctl.before = before;
                            ctl.take_last = take_last || (owner == (int)rank && in_warp < 0);
                            ctl.in_warp = owner != (int)rank ? -1 : in_warp < 0 ? last : in_warp;
                        }
                    } else if (cmd != kEnd) {
                        if (need == kNothing) need = kFinal;
                    }
                    if (lane == 0) {
                        if (cmd == kMass) {
                            ctl.pass = need == kExact ? 0 : need == kRest ? d.k + 1 : d.k;
                        }
                        ctl.d = d;
                        ctl.z = z;
                        ctl.away = away;
                        ctl.left = left;
                        ctl.tried = tried;
                        ctl.exact = exact;
                        ctl.have_mass = have_mass;
                        ctl.need = need;
                    }
                }
                if (child >= 0) {
                    // the child's own first child (for the prefetch), its place in the path
                    const unsigned f0 = __ballot_sync(0xffffffffu, lane > child && lane < n && s_par[lane] == child);
                    const unsigned f1 = __ballot_sync(0xffffffffu, lane + 32 > child && lane + 32 < n && s_par[lane + 32] == child);
                    if (lane == 0) {
                        ctl.cur = child;
                        ctl.ahead = n_path + 1 >= p.M ? -1 : f0 ? __ffs(f0) - 1 : f1 ? __ffs(f1) + 31 : -1;
                        s_path[n_path] = child;
                    }
                }
                if (lane == 0) ctl.cmd = cmd;
            }
            __syncthreads();
            if (ctl.cmd != kMass) break;

            // ---- a mass pass: the sum of every vector's r_pass to my_sum, of the warp's part to s_mass
            double sum = 0.0;
            for (int ch = 0; ch < n_chunks; ++ch) {
                const int vc = v0 + cap * ch, ve = min(vc + cap, v1);
                sum += chunk_mass<LT>(ctl, row, vc, ve, lane, n_chunks > 1, my_row, my_sum, s_table, s_tok);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) s_mass[warp] = sum;
            __syncthreads();
        }
        const int cmd = ctl.cmd;
        if (cmd == kGo) {
            ++n_path;
            enter(ctl.cur);
            continue;
        }
        if (cmd == kSearch) {
            next = -2;                                             // (some warp of the cluster writes the token)
            if (ctl.in_warp == warp) {
                // in index order through the warp's vectors: the first one at whose end the running sum exceeds the target
                // (or the last one that holds anything), then through its elements
                const double target = ctl.target;
                bool take_last = ctl.take_last;
                double run_sum = ctl.before, upto = 0.0;           // upto: the running sum in front of the vector
                int vec = -1;
                bool done = false;
                for (int ch = 0; ch < n_chunks && !done; ++ch) {
                    const int vc = v0 + cap * ch, ve = min(vc + cap, v1);
                    if (n_chunks > 1) chunk_mass<LT>(ctl, row, vc, ve, lane, true, my_row, my_sum, s_table, s_tok);
                    for (int vb = vc; vb < ve && !done; vb += 32) {
                        const double own = vb + lane < ve ? my_sum[vb - vc] : 0.0;
                        double incl = own;
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const double up = __shfl_up_sync(0xffffffffu, incl, o);
                            if (lane >= o) incl += up;
                        }
                        const unsigned any = __ballot_sync(0xffffffffu, own > 0.0);
                        const unsigned hit = take_last ? 0u : __ballot_sync(0xffffffffu, own > 0.0 && run_sum + incl > target);
                        if (hit | any) {
                            const int at = hit ? __ffs(hit) - 1 : 31 - __clz(any);
                            vec = vb + at;                         // (without a hit: the last one so far)
                            upto = run_sum + shfl_d(incl - own, at);
                        }
                        done = hit != 0;
                        run_sum += shfl_d(incl, 31);
                    }
                }
                take_last |= !done;                                // no vector ends beyond the target: the last one's last token
                next = -1;
                if (vec >= 0 && lane == 0) {
                    const int i0 = row.first(vec);
                    double acc = upto;
#pragma unroll 1
                    for (int k = 0; k < N; ++k) {
                        const int i = i0 + k;
                        if (i < 0 || i >= p.V) continue;
                        bool out = false;
                        for (unsigned long long t = ctl.tried; t; t &= t - 1) out |= s_tok[__ffsll((long long)t) - 1] == i;
                        if (out) continue;
                        const float l = Logit<LT>::one(row_ptr + i);
                        double f = weight(!ctl.infinite ? l : l == CUDART_INF_F ? 0.f : -CUDART_INF_F, ctl.d, s_table);
                        if (ctl.pass > 0) f = left_of(f, (double)q_row[i], ctl.pass, ctl.s[0], ctl);
                        if (!(f > 0.0)) continue;
                        next = i;                                  // (the last positive one so far)
                        acc += f;
                        if (!take_last && acc > target) break;
                    }
                }
                if (lane == 0) p.next_token[b] = next;
            }
        }
        break;
    }
    // the path, and the token of greedy requests and of rows that leave nothing (-1)
    if (rank == 0 && warp == 0) {
        for (int i = lane; i < p.M; i += 32) p.path[(long long)b * p.M + i] = i < n_path ? s_path[i] : -1;
        if (lane == 0) {
            p.n_commit[b] = n_path;
            if (ctl.cmd == kEnd) p.next_token[b] = next;
        }
    }
}

template <typename LT, int THREADS>
static cudaError_t launch_verify_as(const VerifyParams &p, int batch, int C, cudaStream_t st)
{
    constexpr int WARPS = THREADS / 32;
    const int vecs = (p.V + 2 * (Logit<LT>::N - 1)) / Logit<LT>::N;               // of an unaligned row
    const int per_warp = (vecs + C * WARPS - 1) / (C * WARPS);
    int cap = (per_warp + 31) / 32 * 32;
    constexpr int most = (int)((size_t)(THREADS == 512 ? 208 : 100) * 1024 / (WARPS * 24)) / 32 * 32;   // one or two thread blocks per SM
    if (cap > most) cap = most;
    const size_t smem = (size_t)WARPS * cap * 24;
    if (cudaError_t e = allow_dynamic_shared(reinterpret_cast<const void *>(verify_tree_kernel<LT, THREADS>), (int)smem)) return e;
    prefer_max_shared_carveout(verify_tree_kernel<LT, THREADS>);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(batch * C));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, verify_tree_kernel<LT, THREADS>, p, C, cap);
}

// Clusters of `size` thread blocks that run at the same time with one block per SM (a cluster stays within one of the GPU's
// processing clusters, whose SM counts need not be a multiple of its size).  Asked once per device and size.
int clusters_at_once(int size)
{
    constexpr int kDevices = 64;
    static std::mutex lock;
    static int known[kDevices][kVerMaxCluster + 1] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= kDevices) {
        cudaGetLastError();
        return sm_count() / (size + 1);
    }
    std::lock_guard<std::mutex> guard(lock);
    if (known[dev][size] == 0) {
        const auto kernel = verify_tree_kernel<float, 512>;
        const int smem = 200 * 1024;                           // one block per SM
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)size;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(size * 1024));
        cfg.blockDim = dim3(512);
        cfg.dynamicSmemBytes = (size_t)smem;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (allow_dynamic_shared(reinterpret_cast<const void *>(kernel), smem) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            n = sm_count() / (size + 1);
        }
        known[dev][size] = n < 1 ? 1 : n;
    }
    return known[dev][size];
}

// The thread blocks of a request: as many as let all requests run at once, at most eight, with 2,048 tokens or more each.
// Where all requests' clusters fit with one block per SM, blocks have 512 threads, else 256 with two blocks per SM.
// (One request, 64-node tree, 151,936 tokens: 512 threads 21 us, 256 threads 28 us.  16 requests, whose clusters of eight do
// not all fit alone: 8 blocks of 256 threads 29 us, 8 of 512 threads 33 us, 7 of 512 threads 30 us.  128 requests, 50,257
// tokens: 2 blocks of 256 threads 31 us, 1 of 512 threads 43 us.)
template <typename LT>
static cudaError_t launch_verify(const VerifyParams &p, int batch, cudaStream_t st)
{
    int C = kVerMaxCluster;
    while (C > 1 && p.V < C * 2048) C >>= 1;
    if (batch <= clusters_at_once(C)) return launch_verify_as<LT, 512>(p, batch, C, st);
    while (C > 1 && (long long)batch * C > 2ll * sm_count()) C >>= 1;
    return launch_verify_as<LT, 256>(p, batch, C, st);
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
    if (batch == 0) return OASIS_OK;
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
    VerifyParams p;
    p.logits = logits; p.tokens = tokens; p.parent = parent; p.n_nodes = n_nodes; p.uniforms = uniforms;
    p.temperature = temperature; p.draft = draft_probs; p.path = path; p.n_commit = n_commit; p.next_token = next_token;
    p.err = error_word();
    p.lb = logits_batch_stride; p.lr = logits_row_stride; p.db = draft_batch_stride; p.dr = draft_row_stride;
    p.T = n_tree; p.V = vocab; p.M = max_path;
    cudaError_t e;
    if (logits_type == OASIS_F32) e = launch_verify<float>(p, batch, (cudaStream_t)stream);
    else if (logits_type == OASIS_BF16) e = launch_verify<__nv_bfloat16>(p, batch, (cudaStream_t)stream);
    else e = launch_verify<__half>(p, batch, (cudaStream_t)stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(OASIS_ERR_CUDA, "%s: launch: %s", who, cudaGetErrorString(e));
    }
    return check_launch(who);
}
