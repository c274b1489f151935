// Scores of given tokens from their logits, and the gradient of the scores.
//
// Forward, one pass over a row z of V logits: a thread keeps the running maximum m of its elements and
//   s = sum e^(z - m),   u = sum e^(z - m) (z - m)            (u <= 0: one sign, no cancellation)
// and rescales both when m grows: with d = m - m', s' = s e^d, u' = (u + s d) e^d.  Threads, then the CTAs of a cluster that
// share a row, are joined by the same rule.  Then
//   lse = m + log s,   log p_v = (z_v - m) - log s,   entropy = log s - u / s.
// A masked entry (-inf) has e^(z - m) = 0; z - m is clamped at -1000, where e^ is 0 in fp32, so that 0 * inf never appears.
//
// The top alternatives cost no second pass: every thread's m is the largest of its elements, so the k-th largest of the
// maxima of disjoint groups of threads is a lower bound for the k-th largest logit.  Only the few threads whose m reaches that
// bound hold candidates, and only their elements are read again (from L2).  Equal logits are ordered by index through
// 64-bit keys (value, ~index), which makes the result independent of the order in which candidates are found.
//
// Backward: dz = g_lp ([v = id] - p) - g_H p (log p + H), element by element from lse and the entropy.
#include "qnn_types.cuh"

namespace qnn {
namespace {

constexpr int MAX_TOP = 32;
constexpr int CAND = 1024;            // candidates a CTA can hold; more (masses of equal logits) take the slow exact path
constexpr float LOG2E = 1.4426950408889634f;
constexpr float FAR = -1000.0f;       // e^-1000 is 0 in fp32
constexpr uint32_t INF_BITS = 0x7f800000u;

__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fc00000u); }
__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// order-preserving map of floats to unsigned: -inf < ... < +inf < NaN, and -0 = +0
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t k)
{
    if (k == 0xffffffffu) return quiet_nan();
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

// A row seen as 16-byte granules of memory: granule i covers elements i * E - shift ... + E - 1; the first and the last may
// be partly outside the row.
template <typename T>
struct Granules {
    static constexpr int E = 16 / (int)sizeof(T);
    const T *row;
    int32_t shift;
    int32_t V;
    __device__ __forceinline__ Granules(const T *r, int32_t v) : row(r), V(v)
    {
        shift = (int32_t)((reinterpret_cast<uintptr_t>(r) & 15u) / sizeof(T));
    }
    __device__ __forceinline__ int64_t count() const { return ((int64_t)V + shift + E - 1) / E; }
    __device__ __forceinline__ int64_t first(int64_t g) const { return g * E - shift; }
    // raw words of granule g; elements outside the row read as -inf and are not touched
    __device__ __forceinline__ uint4 load(int64_t g) const
    {
        const int64_t v0 = first(g);
        if (v0 >= 0 && v0 + E <= V) return *reinterpret_cast<const uint4 *>(row + v0);
        alignas(16) T t[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            t[i] = T(neg_inf());
            if (v0 + i >= 0 && v0 + i < V) t[i] = row[v0 + i];
        }
        return *reinterpret_cast<const uint4 *>(t);
    }
    static __device__ __forceinline__ void floats(const uint4 &w, float (&f)[E])
    {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack2(x[i], f[2 * i], f[2 * i + 1], T());
        }
    }
};

struct Stats {
    float m, s, u;
};
__device__ __forceinline__ void rescale(Stats &a, float to)
{
    const float d = fmaxf(a.m - to, FAR);
    const float c = exp2_approx(d * LOG2E);
    a.u = (a.u + a.s * d) * c;
    a.s *= c;
    a.m = to;
}
__device__ __forceinline__ Stats join(Stats a, Stats b)
{
    const float m = max_nan(a.m, b.m);
    if (m == neg_inf()) return a;
    rescale(a, m);
    rescale(b, m);
    a.s += b.s;
    a.u += b.u;
    return a;
}

struct ScoreArgs {
    const void *logits;
    int64_t ldl;
    int32_t V;
    const int64_t *ids;
    float *logprob, *entropy, *lse;
    int topk;
    float *top_logprob;
    int64_t *top_ids;
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_barrier() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_addr(const void *p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float peer_f32(uint32_t a)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long peer_u64(uint32_t a)
{
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}

template <int THREADS>
struct ScoreShared {
    Stats part[THREADS / 32];
    Stats mine;                                     // this CTA's statistics, read by the cluster's first CTA
    unsigned long long best[MAX_TOP];               // this CTA's largest keys, falling; 0 = none
    unsigned long long cand[CAND];
    uint32_t group[64];
    int flagged[THREADS];
    int n_flagged, n_cand;
    uint32_t bound;
    unsigned long long round_best[THREADS / 32];
};

// The topk largest keys of `n` candidates into out[0..topk), falling; keys are distinct, so every rank is taken once.
template <int THREADS>
__device__ __forceinline__ void rank_candidates(const unsigned long long *cand, int n, int topk, unsigned long long *out)
{
    for (int c = threadIdx.x; c < n; c += THREADS) {
        const unsigned long long k = cand[c];
        if (k == 0ull) continue;
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += cand[j] > k;
        if (rank < topk) out[rank] = k;
    }
}

template <typename T, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) scores_kernel(const ScoreArgs p)
{
    using G = Granules<T>;
    constexpr int E = G::E;
    __shared__ ScoreShared<THREADS> sh;
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t csize = cluster_size(), crank = cluster_rank();
    const int64_t t = blockIdx.x / csize;
    const G row(static_cast<const T *>(p.logits) + t * p.ldl, p.V);
    // this CTA's granules
    const int64_t all = row.count(), per = (all + csize - 1) / csize;
    const int64_t g0 = per * crank < all ? per * crank : all;
    const int64_t g1 = g0 + per < all ? g0 + per : all;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    Stats a = {neg_inf(), 0.0f, 0.0f};
    for (int64_t g = g0 + tid; g < g1; g += (int64_t)THREADS * U) {
        uint4 w[U];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (g + (int64_t)j * THREADS < g1) w[j] = row.load(g + (int64_t)j * THREADS);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (g + (int64_t)j * THREADS >= g1) break;
            float f[E];
            G::floats(w[j], f);
            float b = f[0];
#pragma unroll
            for (int i = 1; i < E; ++i) b = max_nan(b, f[i]);
            if (!(b <= a.m)) rescale(a, max_nan(a.m, b));
            if (a.m == neg_inf()) continue;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float x = fmaxf(f[i] - a.m, FAR);
                const float e = exp2_approx(x * LOG2E);
                a.s += e;
                a.u = fmaf(e, x, a.u);
            }
        }
    }
    const float mine = a.m;                          // the largest of this thread's elements
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Stats b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
        b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
        b.u = __shfl_xor_sync(0xffffffffu, a.u, o);
        // (lower lane first on both sides, so that all lanes hold the same bits)
        a = (lane & o) ? join(b, a) : join(a, b);
    }
    if (lane == 0) sh.part[warp] = a;

    const int topk = p.topk;
    if (topk > 0) {
        constexpr int GL = THREADS >= 512 ? 8 : 4;   // lanes a group: THREADS / GL groups, at least MAX_TOP of them
        constexpr int NG = THREADS / GL;
        static_assert(NG >= MAX_TOP && NG <= 64, "groups");
        float gm = mine;
#pragma unroll
        for (int o = GL / 2; o > 0; o >>= 1) gm = max_nan(gm, __shfl_xor_sync(0xffffffffu, gm, o));
        if ((lane & (GL - 1)) == 0) sh.group[tid / GL] = order_key(gm);
        if (tid == 0) { sh.n_flagged = 0; sh.n_cand = 0; }
        if (tid < MAX_TOP) sh.best[tid] = 0ull;
        __syncthreads();
        if (tid < NG) {                              // the group maximum of rank topk - 1 (ties by group number)
            const uint32_t k = sh.group[tid];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < NG; ++j) rank += (sh.group[j] > k) || (sh.group[j] == k && j < tid);
            if (rank == topk - 1) sh.bound = k;
        }
        __syncthreads();
        const uint32_t bound = sh.bound;
        if (g0 + tid < g1 && order_key(mine) >= bound) sh.flagged[atomicAdd(&sh.n_flagged, 1)] = tid;
        __syncthreads();
        const int nf = sh.n_flagged;
        for (int f = warp; f < nf; f += THREADS / 32) {
            for (int64_t g = g0 + sh.flagged[f] + (int64_t)lane * THREADS; g < g1; g += (int64_t)32 * THREADS) {
                float z[E];
                G::floats(row.load(g), z);
                const int64_t v0 = row.first(g);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int64_t v = v0 + i;
                    const uint32_t k = order_key(z[i]);
                    if (k >= bound && v >= 0 && v < p.V) {
                        const int at = atomicAdd(&sh.n_cand, 1);
                        if (at < CAND) sh.cand[at] = ((unsigned long long)k << 32) | (uint32_t)~(uint32_t)v;
                    }
                }
            }
        }
        __syncthreads();
        if (sh.n_cand <= CAND) {
            rank_candidates<THREADS>(sh.cand, sh.n_cand, topk, sh.best);
        } else {
            // Masses of equal logits at the bound (a row almost wholly masked, a constant row): topk passes, each
            // finding the largest key below the last one.
            unsigned long long last = ~0ull;
            for (int j = 0; j < topk; ++j) {
                unsigned long long b = 0ull;
                for (int64_t g = g0 + tid; g < g1; g += THREADS) {
                    float z[E];
                    G::floats(row.load(g), z);
                    const int64_t v0 = row.first(g);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const int64_t v = v0 + i;
                        const unsigned long long k = ((unsigned long long)order_key(z[i]) << 32) | (uint32_t)~(uint32_t)v;
                        if (v >= 0 && v < p.V && k < last && k > b) b = k;
                    }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long c = __shfl_xor_sync(0xffffffffu, b, o);
                    b = c > b ? c : b;
                }
                if (lane == 0) sh.round_best[warp] = b;
                __syncthreads();
                b = 0ull;
                for (int w = 0; w < THREADS / 32; ++w) b = sh.round_best[w] > b ? sh.round_best[w] : b;
                if (tid == 0) sh.best[j] = b;
                last = b;
                __syncthreads();
                if (b == 0ull) break;                // fewer than topk elements in this CTA's part
            }
        }
    }
    __syncthreads();
    a = sh.part[0];
    for (int w = 1; w < THREADS / 32; ++w) a = join(a, sh.part[w]);

    if (csize > 1) {
        if (tid == 0) sh.mine = a;
        cluster_barrier();
        if (crank == 0) {
            if (topk > 0) {                          // the CTAs' lists side by side
                for (int c = tid; c < (int)csize * topk; c += THREADS) {
                    const int r = c / topk;
                    sh.cand[c] = peer_u64(peer_addr(&sh.best[c - r * topk], (uint32_t)r));
                }
            }
            for (uint32_t r = 1; r < csize; ++r) {
                const uint32_t at = peer_addr(&sh.mine, r);
                const Stats b = {peer_f32(at), peer_f32(at + 4), peer_f32(at + 8)};
                a = join(a, b);
            }
            if (topk > 0) {
                __syncthreads();
                rank_candidates<THREADS>(sh.cand, (int)csize * topk, topk, sh.best);
                __syncthreads();
            }
        }
        cluster_barrier();                           // nobody leaves while its shared memory is being read
        if (crank != 0) return;
    }

    const bool none = a.m == neg_inf();              // a row with nothing left
    const bool bad = !(a.m < __uint_as_float(INF_BITS));
    const float logs = logf(a.s);
    auto logp = [&](float z) { return bad ? quiet_nan() : none ? neg_inf() : (z - a.m) - logs; };
    if (tid == 0) {
        if (p.lse) p.lse[t] = bad ? quiet_nan() : none ? neg_inf() : a.m + logs;
        if (p.entropy) p.entropy[t] = bad ? quiet_nan() : none ? 0.0f : logs - a.u / a.s;
        if (p.logprob) {
            const int64_t id = p.ids[t];
            p.logprob[t] = (id >= 0 && id < p.V) ? logp(to_float(row.row[id])) : 0.0f;
        }
    }
    if (tid < topk) {
        const unsigned long long k = sh.best[tid];
        if (p.top_logprob) p.top_logprob[t * topk + tid] = logp(order_value((uint32_t)(k >> 32)));
        if (p.top_ids) p.top_ids[t * topk + tid] = (int64_t)(uint32_t)~(uint32_t)k;
    }
}

struct ScoreGradArgs {
    const void *logits;
    int64_t ldl;
    int32_t V;
    const int64_t *ids;
    const float *lse, *entropy, *g_logprob, *g_entropy;
    void *d;
    int64_t ldd;
    uint32_t parts;                 // CTAs a row
};

constexpr int GRAD_THREADS = 256, GRAD_U = 4;

// VEC: logits and gradient rows lie alike modulo 16 bytes, so a granule of one is a granule of the other
template <typename T, bool VEC>
__global__ void __launch_bounds__(GRAD_THREADS) scores_grad_kernel(const ScoreGradArgs p)
{
    using G = Granules<T>;
    constexpr int E = G::E;
    griddep_launch_dependents();
    griddep_wait();
    const int64_t t = blockIdx.x / p.parts;
    const uint32_t part = blockIdx.x - (uint32_t)t * p.parts;
    const G row(static_cast<const T *>(p.logits) + t * p.ldl, p.V);
    T *dst = static_cast<T *>(p.d) + t * p.ldd;
    const float lse = p.lse[t];
    const float gh = p.g_entropy ? p.g_entropy[t] : 0.0f, h = p.g_entropy ? p.entropy[t] : 0.0f;
    const int64_t id = p.g_logprob ? p.ids[t] : -1;
    const float gl = (id >= 0 && id < p.V) ? p.g_logprob[t] : 0.0f;
    const bool none = lse == neg_inf();
    const float c = fmaf(gh, h, gl);                 // dz = -p (c + g_H log p), plus g_lp at the token
    auto grad = [&](float z, int64_t v) {
        if (none || z == neg_inf()) return 0.0f;
        const float x = fmaxf(z - lse, FAR);
        const float pr = exp2_approx(x * LOG2E);
        float d = -pr * fmaf(gh, x, c);
        if (v == id) d += gl;
        return lse != lse ? lse : d;
    };
    if (VEC) {
        const int64_t all = row.count(), base = (int64_t)part * (GRAD_THREADS * GRAD_U) + threadIdx.x;
        uint4 w[GRAD_U];
#pragma unroll
        for (int j = 0; j < GRAD_U; ++j)
            if (base + j * GRAD_THREADS < all) w[j] = row.load(base + j * GRAD_THREADS);
#pragma unroll
        for (int j = 0; j < GRAD_U; ++j) {
            const int64_t g = base + j * GRAD_THREADS;
            if (g >= all) break;
            const int64_t v0 = row.first(g);
            float f[E];
            G::floats(w[j], f);
#pragma unroll
            for (int i = 0; i < E; ++i) f[i] = grad(f[i], v0 + i);
            if (v0 >= 0 && v0 + E <= p.V) {
                if constexpr (E == 8) store_floats<T, 8>(dst + v0, f);
                else *reinterpret_cast<float4 *>(dst + v0) = make_float4(f[0], f[1], f[2], f[3]);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (v0 + i >= 0 && v0 + i < p.V) from_float(f[i], dst[v0 + i]);
            }
        }
    } else {
        const int64_t v1 = (int64_t)(part + 1) * (GRAD_THREADS * GRAD_U * E);
        for (int64_t v = (int64_t)part * (GRAD_THREADS * GRAD_U * E) + threadIdx.x; v < v1 && v < p.V; v += GRAD_THREADS)
            from_float(grad(to_float(row.row[v]), v), dst[v]);
    }
}

template <typename T, int THREADS, int U>
int launch_scores_cfg(const ScoreArgs &p, int64_t T_rows, int cluster, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(T_rows * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    unsigned na = 0;
    attr[na].id = cudaLaunchAttributeClusterDimension;
    attr[na].val.clusterDim.x = (unsigned)cluster; attr[na].val.clusterDim.y = 1; attr[na].val.clusterDim.z = 1;
    ++na;
    if (pdl_enabled()) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    cfg.attrs = attr; cfg.numAttrs = na;
    QNN_CUDA(cudaLaunchKernelEx(&cfg, scores_kernel<T, THREADS, U>, p));
    return check_launch("qnn_token_logprobs");
}

template <typename T>
int launch_scores(const ScoreArgs &p, int64_t rows, cudaStream_t st)
{
    const int64_t granules = (int64_t)p.V / Granules<T>::E + 1;
    // Short rows: small blocks, several rows to an SM.  Few long rows: a cluster of CTAs shares a row.
    if (granules <= 512) return launch_scores_cfg<T, 128, 4>(p, rows, 1, st);
    int cluster = 1;
    while (cluster < 8 && rows * cluster * 2 <= 2 * (int64_t)sm_count() && granules / (cluster * 2) >= 512) cluster *= 2;
    return launch_scores_cfg<T, 512, 4>(p, rows, cluster, st);
}

template <typename T>
int launch_scores_grad(ScoreGradArgs p, int64_t rows, cudaStream_t st)
{
    constexpr int E = Granules<T>::E;
    const int64_t granules = (int64_t)p.V / E + 2;
    p.parts = (uint32_t)ceil_div(granules, GRAD_THREADS * GRAD_U);
    const bool vec = (reinterpret_cast<uintptr_t>(p.logits) & 15u) == (reinterpret_cast<uintptr_t>(p.d) & 15u) &&
                     (p.ldl * (int64_t)sizeof(T)) % 16 == (p.ldd * (int64_t)sizeof(T)) % 16;
    QNN_REQUIRE(rows * (int64_t)p.parts < ((int64_t)1 << 31), QNN_ERR_UNSUPPORTED, "qnn_token_logprobs_backward: too many elements for one launch");
    const dim3 grid((unsigned)(rows * p.parts));
    if (vec) QNN_CUDA(launch_pdl(scores_grad_kernel<T, true>, grid, dim3(GRAD_THREADS), 0, st, p));
    else QNN_CUDA(launch_pdl(scores_grad_kernel<T, false>, grid, dim3(GRAD_THREADS), 0, st, p));
    return check_launch("qnn_token_logprobs_backward");
}

int check_logits(const char *what, const void *logits, int type, int64_t T, int64_t V, int64_t ldl)
{
    QNN_REQUIRE(type_ok(type), QNN_ERR_INVALID_ARG, "%s: unknown element type %d", what, type);
    QNN_REQUIRE(T >= 0 && V >= 0, QNN_ERR_INVALID_ARG, "%s: negative size", what);
    QNN_REQUIRE(V < ((int64_t)1 << 31) - 64 && T < ((int64_t)1 << 28), QNN_ERR_UNSUPPORTED, "%s: V of 2^31 or T of 2^28 and more", what);
    if (T == 0) return QNN_OK;
    QNN_REQUIRE(V >= 1, QNN_ERR_INVALID_ARG, "%s: V is 0", what);
    QNN_REQUIRE(logits != nullptr, QNN_ERR_INVALID_ARG, "%s: logits is NULL", what);
    QNN_REQUIRE(ldl >= V, QNN_ERR_INVALID_ARG, "%s: ldl below V", what);
    QNN_REQUIRE(aligned(logits, (size_t)type_bytes(type)), QNN_ERR_ALIGNMENT, "%s: logits are not aligned to their elements", what);
    return QNN_OK;
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

int qnn_token_logprobs(const void *logits, int type, int64_t T, int64_t V, int64_t ldl, const int64_t *ids, float *logprob, float *entropy,
                       float *lse, int topk, float *top_logprob, int64_t *top_ids, void *stream)
{
    const char *what = "qnn_token_logprobs";
    if (int rc = check_logits(what, logits, type, T, V, ldl)) return rc;
    QNN_REQUIRE(topk >= 0, QNN_ERR_INVALID_ARG, "%s: topk is negative", what);
    QNN_REQUIRE(topk <= MAX_TOP, QNN_ERR_UNSUPPORTED, "%s: at most %d alternatives", what, MAX_TOP);
    if (T == 0) return QNN_OK;
    QNN_REQUIRE(topk <= V, QNN_ERR_INVALID_ARG, "%s: topk above V", what);
    QNN_REQUIRE(logprob == nullptr || ids != nullptr, QNN_ERR_INVALID_ARG, "%s: logprob needs ids", what);
    QNN_REQUIRE(topk == 0 || top_logprob || top_ids, QNN_ERR_INVALID_ARG, "%s: topk without an output for it", what);
    QNN_REQUIRE(logprob || entropy || lse || topk > 0, QNN_ERR_INVALID_ARG, "%s: no output asked for", what);
    QNN_REQUIRE(aligned(ids, 8) && aligned(top_ids, 8) && aligned(logprob, 4) && aligned(entropy, 4) && aligned(lse, 4) && aligned(top_logprob, 4),
                QNN_ERR_ALIGNMENT, "%s: a pointer is not aligned to its elements", what);
    ScoreArgs p{};
    p.logits = logits; p.ldl = ldl; p.V = (int32_t)V;
    p.ids = ids; p.logprob = logprob; p.entropy = entropy; p.lse = lse;
    p.topk = topk; p.top_logprob = top_logprob; p.top_ids = top_ids;
    cudaStream_t st = as_stream(stream);
    switch (type) {
        case QNN_TYPE_F32: return launch_scores<float>(p, T, st);
        case QNN_TYPE_BF16: return launch_scores<__nv_bfloat16>(p, T, st);
        default: return launch_scores<__half>(p, T, st);
    }
}

int qnn_token_logprobs_backward(const void *logits, int type, int64_t T, int64_t V, int64_t ldl, const int64_t *ids, const float *lse,
                                const float *entropy, const float *g_logprob, const float *g_entropy, void *d_logits, int64_t ldd, void *stream)
{
    const char *what = "qnn_token_logprobs_backward";
    if (int rc = check_logits(what, logits, type, T, V, ldl)) return rc;
    if (T == 0) return QNN_OK;
    QNN_REQUIRE(lse && d_logits, QNN_ERR_INVALID_ARG, "%s: NULL pointer", what);
    QNN_REQUIRE(g_logprob || g_entropy, QNN_ERR_INVALID_ARG, "%s: no incoming gradient", what);
    QNN_REQUIRE(!g_logprob || ids, QNN_ERR_INVALID_ARG, "%s: g_logprob needs ids", what);
    QNN_REQUIRE(!g_entropy || entropy, QNN_ERR_INVALID_ARG, "%s: g_entropy needs the entropy", what);
    QNN_REQUIRE(ldd >= V, QNN_ERR_INVALID_ARG, "%s: ldd below V", what);
    QNN_REQUIRE(d_logits != logits || ldd == ldl, QNN_ERR_INVALID_ARG, "%s: a gradient over the logits needs the same leading dimension", what);
    QNN_REQUIRE(aligned(d_logits, (size_t)type_bytes(type)) && aligned(ids, 8) && aligned(lse, 4) && aligned(entropy, 4) && aligned(g_logprob, 4) &&
                    aligned(g_entropy, 4),
                QNN_ERR_ALIGNMENT, "%s: a pointer is not aligned to its elements", what);
    ScoreGradArgs p{};
    p.logits = logits; p.ldl = ldl; p.V = (int32_t)V;
    p.ids = ids; p.lse = lse; p.entropy = entropy; p.g_logprob = g_logprob; p.g_entropy = g_entropy;
    p.d = d_logits; p.ldd = ldd;
    cudaStream_t st = as_stream(stream);
    switch (type) {
        case QNN_TYPE_F32: return launch_scores_grad<float>(p, T, st);
        case QNN_TYPE_BF16: return launch_scores_grad<__nv_bfloat16>(p, T, st);
        default: return launch_scores_grad<__half>(p, T, st);
    }
}

}  // extern "C"
