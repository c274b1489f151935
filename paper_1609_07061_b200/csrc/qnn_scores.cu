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
#include <type_traits>
#include <atomic>
#include "qnn_types.cuh"
#include "qnn_tc_ptx.cuh"

namespace qnn {
namespace {

constexpr int MAX_TOP = 32;
constexpr int MAX_CLUSTER = 8;        // CTAs that share a row
constexpr int CAND = 256;             // candidates a CTA can hold; more (masses of equal logits) take the slow exact path
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
    __device__ __forceinline__ int32_t count() const { return (V + shift + E - 1) / E; }
    __device__ __forceinline__ int32_t first(int32_t g) const { return g * E - shift; }
    // granules first_full() .. end_full() - 1 lie wholly inside the row
    __device__ __forceinline__ int32_t first_full() const { return shift > 0; }
    __device__ __forceinline__ int32_t end_full() const { return (V + shift) / E; }
    __device__ __forceinline__ const uint4 *at(int32_t g) const { return reinterpret_cast<const uint4 *>(row + first(g)); }
    // any granule: elements outside the row read as -inf and are not touched
    __device__ __forceinline__ uint4 load(int32_t g) const
    {
        if (g >= first_full() && g < end_full()) return *at(g);
        const int32_t v0 = first(g);
        alignas(16) T t[E];
#pragma unroll 1
        for (int i = 0; i < E; ++i) t[i] = (v0 + i >= 0 && v0 + i < V) ? row[v0 + i] : T(neg_inf());
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

// Below this magnitude of the reference (the running maximum, or lse) the element loops clamp the LOGITS at -2^60 (f16: at
// its lowest value) instead of the differences: on packed 16-bit pairs that is half an instruction an element, e^ of such an
// element is 0 all the same, and its difference stays finite.  References beyond it take the plain loops.
// (f16 has no room below its lowest value: the reference must be well above it for e^ of a clamped element to be 0.)
template <typename T>
__device__ __forceinline__ bool calm_at(float ref)
{
    if (std::is_same<T, __half>::value) return ref > -64000.0f && ref < 1e15f;
    return fabsf(ref) < 1e15f;
}

// largest of the 16-bit pairs of two words (a NaN stays), and the clamp
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b, __nv_bfloat16)
{
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b, __half)
{
    const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b, float) { return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b))); }
__device__ __forceinline__ float top_of(uint32_t w, float) { return __uint_as_float(w); }
template <typename T>
__device__ __forceinline__ float top_of(uint32_t w, T)
{
    float lo, hi;
    unpack2(w, lo, hi, T());
    return max_nan(lo, hi);
}
// the elements of a granule as pairs, clamped
__device__ __forceinline__ void calm_pairs(const uint4 &w, f32x2 (&z)[4], __nv_bfloat16)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    const uint32_t low = 0xDD80DD80u;            // -2^60 twice
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 c = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&x[i]), *reinterpret_cast<const __nv_bfloat162 *>(&low));
        float lo, hi;
        unpack2(*reinterpret_cast<const uint32_t *>(&c), lo, hi, __nv_bfloat16());
        z[i] = pair(lo, hi);
    }
}
__device__ __forceinline__ void calm_pairs(const uint4 &w, f32x2 (&z)[4], __half)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    const uint32_t low = 0xFBFFFBFFu;            // -65504 twice
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 c = __hmax2(*reinterpret_cast<const __half2 *>(&x[i]), *reinterpret_cast<const __half2 *>(&low));
        const float2 f = __half22float2(c);
        z[i] = pair(f.x, f.y);
    }
}
__device__ __forceinline__ void calm_pairs(const uint4 &w, f32x2 (&z)[2], float)
{
    const float low = -1.152921504606846976e18f;  // -2^60
    z[0] = pair(fmaxf(__uint_as_float(w.x), low), fmaxf(__uint_as_float(w.y), low));
    z[1] = pair(fmaxf(__uint_as_float(w.z), low), fmaxf(__uint_as_float(w.w), low));
}

// Running statistics of one thread: m, and s and u as two partial sums each.
struct Running {
    float m;
    f32x2 s, u;
    __device__ __forceinline__ Stats stats() const
    {
        float a, b, c, d;
        unpair(s, a, b);
        unpair(u, c, d);
        return {m, a + b, c + d};
    }
};
// adds N granules (words of elements outside the row are -inf); returns their largest element
template <typename T, int N>
__device__ __forceinline__ float add_granules(Running &a, const uint4 (&w)[N])
{
    constexpr int E = Granules<T>::E;
    uint32_t top = max_words(max_words(w[0].x, w[0].y, T()), max_words(w[0].z, w[0].w, T()), T());
#pragma unroll
    for (int j = 1; j < N; ++j) top = max_words(top, max_words(max_words(w[j].x, w[j].y, T()), max_words(w[j].z, w[j].w, T()), T()), T());
    const float b = top_of(top, T());
    if (!(b <= a.m)) {
        const float to = max_nan(a.m, b);
        const float d = fmaxf(a.m - to, FAR);
        const float c = exp2_approx(d * LOG2E);
        a.u = mul2(fma2(a.s, pair(d, d), a.u), pair(c, c));
        a.s = mul2(a.s, pair(c, c));
        a.m = to;
    }
    if (calm_at<T>(a.m)) {
        const f32x2 nm = pair(-a.m, -a.m), l2e = pair(LOG2E, LOG2E);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            f32x2 z[E / 2];
            calm_pairs(w[j], z, T());
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const f32x2 x = add2(z[i], nm);
                float lo, hi;
                unpair(mul2(x, l2e), lo, hi);
                const f32x2 e = pair(exp2_approx(lo), exp2_approx(hi));
                a.s = add2(a.s, e);
                a.u = fma2(e, x, a.u);
            }
        }
    } else if (a.m != neg_inf()) {
        // (unrolled: a loop over w[j] would put the granules of EVERY call into local memory)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float f[E];
            Granules<T>::floats(w[j], f);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float x = fmaxf(f[i] - a.m, FAR);
                const f32x2 e = pair(exp2_approx(x * LOG2E), 0.0f);
                a.s = add2(a.s, e);
                a.u = fma2(e, pair(x, 0.0f), a.u);
            }
        }
    }
    return b;
}

struct ScoreArgs {
    const void *logits;
    int64_t T, ldl;
    int32_t V;
    const int64_t *ids;
    float *logprob, *entropy, *lse;
    int topk;
    float *top_logprob;
    int64_t *top_ids;
};

__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t peer_addr(const void *p, uint32_t rank) { return map_to_cta(smem_u32(p), rank); }
// asynchronous stores into another CTA's shared memory that report their bytes to a barrier there
__device__ __forceinline__ void send_u64(uint32_t a, unsigned long long v, uint32_t bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.u64 [%0], %1, [%2];" ::"r"(a), "l"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void send_f32x4(uint32_t a, float x, float y, float z, float w, uint32_t bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(a), "f"(x), "f"(y), "f"(z), "f"(w), "r"(bar) : "memory");
}

// THREADS threads add, one more warp loads.  Rows stream through a ring of STAGES chunks of THREADS * U granules in shared
// memory, filled by bulk copies, so that what is in flight does not depend on how far the adding threads are.
template <int THREADS, int U, int STAGES>
struct ScoreShared {
    static constexpr int CHUNK = THREADS * U;       // granules
    static constexpr int GL = THREADS / 32;         // lanes a group: 32 groups of threads
    static_assert(GL >= 2 && GL <= 32 && MAX_TOP <= 32 && MAX_CLUSTER * MAX_TOP <= CAND, "groups");
    uint4 ring[STAGES][CHUNK];
    unsigned long long full[STAGES], empty[STAGES]; // barriers
    int abort_flag;
    int n_cand, n_one, n_all, n_join;
    // in the cluster's first CTA: what every CTA found -- its statistics and at most MAX_TOP keys, 0 = none
    unsigned long long gathered;                    // barrier
    alignas(16) float4 theirs[MAX_CLUSTER];
    unsigned long long theirs_best[MAX_CLUSTER][MAX_TOP];
    alignas(16) uint32_t group[32];                 // largest element of each group of threads, as order keys
    float2 part[THREADS / 32];                      // s and u of each warp
    uint32_t one[THREADS];                          // threads that hold candidates in one chunk: chunk * THREADS + thread
    uint32_t all[THREADS];                          // ... perhaps in several
    unsigned long long best[MAX_TOP];               // this CTA's largest keys, falling; 0 = none
    alignas(16) unsigned long long cand[CAND];
    unsigned long long round_best[THREADS / 32];
};

// The topk largest keys of `n` candidates, each handed with its rank to put(rank, key); keys are distinct (0 = none), so
// every rank is taken once.
template <int THREADS, class Put>
__device__ __forceinline__ void rank_candidates(const unsigned long long *cand, int n, int topk, Put put)
{
    for (int c = threadIdx.x; c < n; c += THREADS) {
        const unsigned long long k = cand[c];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j + 1 < n; j += 2) {
            const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(cand + j);
            rank += (int)(o.x > k) + (int)(o.y > k);
        }
        if ((n & 1) && cand[n - 1] > k) ++rank;
        if (rank < topk && k != 0ull) put(rank, k);
    }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n"
                 "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%2], [%3], %1, [%0];"
                 ::"r"(bar), "r"(bytes), "r"(dst), "l"(src) : "memory");
}
template <int THREADS>
__device__ __forceinline__ void adders_sync() { asm volatile("barrier.sync 1, %0;" ::"n"(THREADS) : "memory"); }

// One CTA (or one cluster of them) a row, RESIDENT CTAs an SM: while one joins its statistics and finds its alternatives, the
// others stream.  (CTAs that walk several rows and load ahead across them were slower, 97 against 90 us on 2048 x 131072
// without alternatives: SMs differ in how fast they stream, and the hardware hands out rows as they finish.)
// SELFTEST: CTA 1 of a cluster ends without sending what it found, CTA 2 sends late, and the first one waits for a short time only.
template <typename T, int THREADS, int U, int STAGES, int RESIDENT, bool SELFTEST = false>
__global__ void __launch_bounds__(THREADS + 32, RESIDENT) scores_kernel(const ScoreArgs p)
{
    using G = Granules<T>;
    using SH = ScoreShared<THREADS, U, STAGES>;
    constexpr int E = G::E;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    SH &sh = *reinterpret_cast<SH *>(smem_raw);
    volatile int *abort_flag = &sh.abort_flag;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&sh.full[s]), 1); mbar_init(smem_u32(&sh.empty[s]), THREADS / 32); }
        mbar_init(smem_u32(&sh.gathered), 1);
        *abort_flag = 0;
        sh.n_cand = 0; sh.n_one = 0; sh.n_all = 0; sh.n_join = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
        // what the CTAs of a cluster send to the first one
        const uint32_t expected = cluster_size() * (16u + (p.topk > 0 ? 8u * MAX_TOP : 0u));
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(&sh.gathered)), "r"(expected) : "memory");
    }
    __syncthreads();
    const uint32_t csize = cluster_size(), crank = csize > 1 ? cluster_ctarank() : 0u;
    if (csize > 1) cluster_arrive();                     // nothing is sent before the first CTA's barrier stands
    griddep_wait();
    const int64_t t = blockIdx.x / csize;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const G row(static_cast<const T *>(p.logits) + t * p.ldl, p.V);
    // this CTA's whole granules of the row
    int32_t g0, g1;
    {
        const int32_t f0 = row.first_full(), n = row.end_full() - f0, share = (n + (int32_t)csize - 1) / (int32_t)csize;
        g0 = f0 + min(share * (int32_t)crank, n);
        g1 = f0 + min(share * ((int32_t)crank + 1), n);
    }
    int stage = 0;
    uint32_t phase = 0;

    if (warp == THREADS / 32) {
        if (lane == 0) {
            for (int32_t g = g0; g < g1; g += SH::CHUNK) {
                if (!mbar_wait(smem_u32(&sh.empty[stage]), phase ^ 1u, abort_flag, 21)) break;
                const int32_t n = min(g1 - g, SH::CHUNK);
                bulk_load(smem_u32(sh.ring[stage]), row.at(g), (uint32_t)(n * 16), smem_u32(&sh.full[stage]));
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
            if (*abort_flag) let_flights_land();
        }
        __syncwarp();
        if (csize > 1) cluster_wait();
        return;
    }

    const int topk = p.topk;
    // the token's logit is on its way while the row streams
    int64_t id = -1;
    float token = 0.0f;
    constexpr int TOKEN = THREADS - 32;              // (not of the first warp, which has the alternatives to rank)
    if (tid == TOKEN && crank == 0 && p.logprob != nullptr) {
        id = p.ids[t];
        if (id >= 0 && id < p.V) token = to_float(row.row[id]);
    }
    Running run = {neg_inf(), 0ull, 0ull};
    float second = neg_inf();                        // the largest element outside this thread's best chunk
    uint32_t best_chunk = 0, chunk = 0;
    for (int32_t g = g0; g < g1; g += SH::CHUNK, ++chunk) {
        // (a wait that runs out raises the status word; the row is then finished on what the ring holds)
        (void)mbar_wait(smem_u32(&sh.full[stage]), phase, abort_flag, 22);
        const int n = min(g1 - g, SH::CHUNK);
        uint4 w[U];
        if (n == SH::CHUNK) {
#pragma unroll
            for (int j = 0; j < U; ++j) w[j] = sh.ring[stage][j * THREADS + tid];
        } else {
            constexpr uint32_t fill = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;   // -inf
#pragma unroll
            for (int j = 0; j < U; ++j) {
                w[j] = make_uint4(fill, fill, fill, fill);
                if (j * THREADS + tid < n) w[j] = sh.ring[stage][j * THREADS + tid];
            }
        }
        // The stage is handed back to a bulk copy, which is of the asynchronous proxy: without this fence it may overtake the reads
        // above.  (It did, where other rows on the SM kept its memory pipe busy with their alternatives: 232 x 171761 fp32 with 32
        // of them, sums of some rows off by 1e-4 to 1e-2.  With it 2048 x 131072 bf16 takes 94.7 us for 94.3, 4 x 128000 6.3 for 6.2.)
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.empty[stage]));
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        const float before = run.m;
        float b = neg_inf();
        if (n > THREADS) {
            b = add_granules<T, U>(run, w);
        } else if (tid < n) {
            const uint4 only[1] = {w[0]};
            b = add_granules<T, 1>(run, only);
        }
        second = fmaxf(second, fminf(before, b));
        if (b > before) best_chunk = chunk;
    }
    // The row is in: the next kernel may be scheduled now.  (Allowed to start at once, its CTAs pile up on the SMs that are
    // still free, several to one, and stay there.)
    griddep_launch_dependents();
    // Granules that the row only shares with its neighbours: the head is thread 0's, the tail thread 1's, of the first
    // CTA.  (A row inside one granule is a head.)
    const bool head = row.first_full() > 0, tail = row.end_full() < row.count() && row.count() > row.first_full();
    const bool has_edge = crank == 0 && ((tid == 0 && head) || (tid == 1 && tail));
    const int32_t edge = tid == 0 ? 0 : row.count() - 1;
    if (has_edge) {
        const uint4 only[1] = {row.load(edge)};
        (void)add_granules<T, 1>(run, only);
    }
    const float mine = run.m;                        // the largest of this thread's elements
    // the row's (or part's) maximum, through the groups' maxima
    float gm = mine;
#pragma unroll
    for (int o = SH::GL / 2; o > 0; o >>= 1) gm = max_nan(gm, __shfl_xor_sync(0xffffffffu, gm, o));
    if ((lane & (SH::GL - 1)) == 0) sh.group[tid / SH::GL] = order_key(gm);
    adders_sync<THREADS>();
    const uint32_t gkey = sh.group[lane];
    Stats a = run.stats();
    {
        const float m = order_value(__reduce_max_sync(0xffffffffu, gkey));
        if (m != neg_inf()) rescale(a, m);           // (all -inf: s and u are 0)
        else a.m = m;
    }
    // s and u of the block: every thread has scaled its own to the common maximum, plain sums are left
    float s = a.s, u = a.u;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        u += __shfl_xor_sync(0xffffffffu, u, o);
    }
    if (lane == 0) sh.part[warp] = make_float2(s, u);
    uint32_t bound = 0u;
    if (topk > 0) {
        // the topk-th largest of the groups' maxima: the smallest one that fewer than topk are above
        int above = 0;
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(&sh.group[j]);
            above += (int)(o.x > gkey) + (int)(o.y > gkey) + (int)(o.z > gkey) + (int)(o.w > gkey);
        }
        bound = __reduce_min_sync(0xffffffffu, above < topk ? gkey : 0xffffffffu);
        // threads that hold candidates: in their best chunk alone, or perhaps elsewhere too
        if (order_key(mine) >= bound) {
            if (order_key(second) >= bound || mine != mine) sh.all[atomicAdd(&sh.n_all, 1)] = (uint32_t)tid;
            else if (run.m > neg_inf()) sh.one[atomicAdd(&sh.n_one, 1)] = best_chunk * THREADS + (uint32_t)tid;
        }
    }
    adders_sync<THREADS>();
    a.s = 0.0f; a.u = 0.0f;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) { a.s += sh.part[i].x; a.u += sh.part[i].y; }

    bool listed = false;                             // the keys stand in sh.best, not in sh.cand
    if (topk > 0) {
        auto offer = [&](const uint4 &words, int32_t v0) {
            float z[E];
            G::floats(words, z);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint32_t k = order_key(z[i]);
                if (k >= bound && v0 + i >= 0 && v0 + i < p.V) {
                    const int at = atomicAdd(&sh.n_cand, 1);
                    if (at < CAND) sh.cand[at] = ((unsigned long long)k << 32) | (uint32_t)~(uint32_t)(v0 + i);
                }
            }
        };
        // a part that fits the ring still stands there (4 x 128000 with 5 alternatives: 6.2 us against 6.7)
        const bool in_ring = g1 - g0 <= STAGES * SH::CHUNK;
        auto granule = [&](int32_t rel) { return in_ring ? sh.ring[0][rel] : *row.at(g0 + rel); };
        const int n_one = sh.n_one * U;
        for (int i = tid; i < n_one; i += THREADS) {
            const uint32_t e = sh.one[i / U], c = e / THREADS;
            const int32_t rel = (int32_t)(c * SH::CHUNK + (i % U) * THREADS + (e - c * THREADS));
            if (rel < g1 - g0) offer(granule(rel), row.first(g0 + rel));
        }
        const uint32_t per = (uint32_t)((g1 - g0 + THREADS - 1) / THREADS);
        const uint32_t n_all = (uint32_t)sh.n_all * per;
        for (uint32_t i = tid; i < n_all; i += THREADS) {
            const uint32_t f = (uint32_t)(i / per);
            const int32_t rel = (int32_t)(sh.all[f] + (i - f * per) * THREADS);
            if (rel < g1 - g0) offer(granule(rel), row.first(g0 + rel));
        }
        if (has_edge && order_key(mine) >= bound) offer(row.load(edge), row.first(edge));
        adders_sync<THREADS>();
        if (sh.n_cand > CAND) {
            // Masses of equal logits at the bound (a row almost wholly masked, a constant row): topk passes, each
            // finding the largest key below the last one.
            listed = true;
            if (tid < MAX_TOP) sh.best[tid] = 0ull;
            unsigned long long last = ~0ull;
            for (int j = 0; j < topk; ++j) {
                unsigned long long b = 0ull;
                auto look = [&](const uint4 &words, int32_t v0) {
                    float z[E];
                    G::floats(words, z);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const int32_t v = v0 + i;
                        const unsigned long long k = ((unsigned long long)order_key(z[i]) << 32) | (uint32_t)~(uint32_t)v;
                        if (v >= 0 && v < p.V && k < last && k > b) b = k;
                    }
                };
                for (int32_t g = g0 + tid; g < g1; g += THREADS) look(*row.at(g), row.first(g));
                if (has_edge) look(row.load(edge), row.first(edge));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long c = __shfl_xor_sync(0xffffffffu, b, o);
                    b = c > b ? c : b;
                }
                adders_sync<THREADS>();
                if (lane == 0) sh.round_best[warp] = b;
                adders_sync<THREADS>();
                b = 0ull;
                for (int i = 0; i < THREADS / 32; ++i) b = sh.round_best[i] > b ? sh.round_best[i] : b;
                if (tid == 0) sh.best[j] = b;
                last = b;
                if (b == 0ull) break;                // fewer than topk elements in this CTA's part
            }
            adders_sync<THREADS>();
        }
    }

    if (*abort_flag) let_flights_land();
    if (csize > 1) {
        // every CTA sends what it found to the first one, which goes on alone: at most MAX_TOP keys each
        int n_mine = topk > 0 ? sh.n_cand : 0;
        if (topk > 0 && !listed && n_mine > MAX_TOP) {
            if (tid < MAX_TOP) sh.best[tid] = 0ull;
            adders_sync<THREADS>();
            rank_candidates<THREADS>(sh.cand, n_mine, topk, [&](int rank, unsigned long long k) { sh.best[rank] = k; });
            adders_sync<THREADS>();
            listed = true;
        }
        if (listed) n_mine = topk;
        __syncwarp();
        cluster_wait();
        if (SELFTEST && crank == 1) return;
        if (SELFTEST && crank == 2)
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        const uint32_t bar = peer_addr(&sh.gathered, 0);
        if (warp == 0) {
            if (topk > 0) send_u64(peer_addr(&sh.theirs_best[crank][lane], 0), lane < n_mine ? (listed ? sh.best[lane] : sh.cand[lane]) : 0ull, bar);
            if (lane == 0) send_f32x4(peer_addr(&sh.theirs[crank], 0), a.m, a.s, a.u, 0.0f, bar);
        }
        if (crank != 0) return;
        (void)mbar_wait(smem_u32(&sh.gathered), 0, abort_flag, 23, SELFTEST ? 64u : WAIT_LIMIT);
        __syncwarp();
        // every warp joins the CTAs' statistics: lane r holds those of CTA r (their number is a power of two)
        const float4 theirs = sh.theirs[lane & (csize - 1)];
        a = {theirs.x, theirs.y, theirs.z};
        for (uint32_t o = 1; o < csize; o <<= 1) {
            Stats b;
            b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
            b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
            b.u = __shfl_xor_sync(0xffffffffu, a.u, o);
            a = (lane & o) ? join(b, a) : join(a, b);    // (the same order on both sides: all lanes hold the same bits)
        }
        listed = false;
        if (topk > 0) {
            // their keys side by side, in any order, over this CTA's own, which have been sent and received
            for (uint32_t r = warp; r < csize; r += THREADS / 32) {
                const unsigned long long k = sh.theirs_best[r][lane];
                const uint32_t have = __ballot_sync(0xffffffffu, k != 0ull);
                int at = 0;
                if (lane == 0) at = atomicAdd(&sh.n_join, __popc(have));
                at = __shfl_sync(0xffffffffu, at, 0);
                if (k != 0ull) sh.cand[at + __popc(have & ((1u << lane) - 1u))] = k;
            }
            adders_sync<THREADS>();
        }
    }

    if (crank == 0) {
        const bool none = a.m == neg_inf();          // a row with nothing left
        const bool bad = !(a.m < __uint_as_float(INF_BITS));
        const float logs = logf(a.s);
        auto logp = [&](float z) { return bad ? quiet_nan() : none ? neg_inf() : (z - a.m) - logs; };
        if (tid == TOKEN) {
            if (p.lse) p.lse[t] = bad ? quiet_nan() : none ? neg_inf() : a.m + logs;
            if (p.entropy) p.entropy[t] = bad ? quiet_nan() : none ? 0.0f : logs - a.u / a.s;
            if (p.logprob) p.logprob[t] = (id >= 0 && id < p.V) ? logp(token) : 0.0f;
        }
        auto put = [&](int rank, unsigned long long k) {
            if (p.top_logprob) p.top_logprob[t * topk + rank] = logp(order_value((uint32_t)(k >> 32)));
            if (p.top_ids) p.top_ids[t * topk + rank] = (int64_t)(uint32_t)~(uint32_t)k;
        };
        if (listed) {
            if (tid < topk) put(tid, sh.best[tid]);
        } else if (topk > 0) {
            rank_candidates<THREADS>(sh.cand, csize > 1 ? sh.n_join : sh.n_cand, topk, put);
        }
        // the others may not have sent everything yet
        if (csize > 1 && __any_sync(0xffffffffu, *abort_flag)) stay_for_cluster();
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
    int32_t span;                   // granules a CTA, whole rounds of GRAD_THREADS * GRAD_U
};

constexpr int GRAD_THREADS = 256, GRAD_U = 4;

struct GradRow {
    float lse, gh, h, gl, c;       // dz = -p (c + g_H log p), plus g_lp at the token
    int64_t id;
    bool none;
    __device__ __forceinline__ float grad(float z, int64_t v) const
    {
        if (none || z == neg_inf()) return 0.0f;
        const float x = fmaxf(z - lse, FAR);
        float d = -exp2_approx(x * LOG2E) * fmaf(gh, x, c);
        if (v == id) d += gl;
        return lse != lse ? lse : d;
    }
};

// VEC: logits and gradient rows lie alike modulo 16 bytes, so a granule of one is a granule of the other
template <typename T, bool VEC>
__global__ void __launch_bounds__(GRAD_THREADS) scores_grad_kernel(const ScoreGradArgs p)
{
    using G = Granules<T>;
    constexpr int E = G::E;
    griddep_wait();
    const int64_t t = blockIdx.x / p.parts;
    const uint32_t part = blockIdx.x - (uint32_t)t * p.parts;
    const G row(static_cast<const T *>(p.logits) + t * p.ldl, p.V);
    T *dst = static_cast<T *>(p.d) + t * p.ldd;
    GradRow r;
    r.lse = p.lse[t];
    r.gh = p.g_entropy ? p.g_entropy[t] : 0.0f;
    r.h = p.g_entropy ? p.entropy[t] : 0.0f;
    r.id = p.g_logprob ? p.ids[t] : -1;
    r.gl = (r.id >= 0 && r.id < p.V) ? p.g_logprob[t] : 0.0f;
    r.none = r.lse == neg_inf();
    r.c = fmaf(r.gh, r.h, r.gl);
    if (VEC) {
        const int32_t f0 = row.first_full(), f1 = row.end_full();
        // the token's place in the row; -E where there is none
        const int32_t id = r.id >= 0 && r.id < p.V ? (int32_t)r.id : -E;
        const bool calm = calm_at<T>(r.lse) && fabsf(r.gh) < 1e15f && fabsf(r.c) < 1e15f;
        const f32x2 nlse = pair(-r.lse, -r.lse), l2e = pair(LOG2E, LOG2E), ngh = pair(-r.gh, -r.gh), nc = pair(-r.c, -r.c);
        const int32_t g1 = min(f1, (int32_t)(part + 1) * p.span);
#pragma unroll 1
        for (int32_t base = (int32_t)part * p.span + (int32_t)threadIdx.x; base < g1; base += GRAD_THREADS * GRAD_U) {
            uint4 w[GRAD_U];
#pragma unroll
            for (int j = 0; j < GRAD_U; ++j) {
                const int32_t g = base + j * GRAD_THREADS;
                if (g >= f0 && g < g1) w[j] = *row.at(g);
            }
#pragma unroll
            for (int j = 0; j < GRAD_U; ++j) {
                const int32_t g = base + j * GRAD_THREADS;
                if (g < f0 || g >= g1) continue;
                const int32_t v0 = row.first(g);
                float f[E];
                if (calm) {
                    f32x2 z[E / 2];
                    calm_pairs(w[j], z, T());
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        const f32x2 x = add2(z[i], nlse);
                        float lo, hi;
                        unpair(mul2(x, l2e), lo, hi);
                        unpair(mul2(pair(exp2_approx(lo), exp2_approx(hi)), fma2(ngh, x, nc)), f[2 * i], f[2 * i + 1]);
                    }
                    const int32_t at = id - v0;
                    if (at >= 0 && at < E) {             // the token's own entry, unless it is masked
                        float z1[E];
                        G::floats(w[j], z1);
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            if (i == at && z1[i] != neg_inf()) f[i] += r.gl;
                    }
                } else {
                    G::floats(w[j], f);
#pragma unroll
                    for (int i = 0; i < E; ++i) f[i] = r.grad(f[i], v0 + i);
                }
                if constexpr (E == 8) store_floats<T, 8>(dst + v0, f);
                else *reinterpret_cast<float4 *>(dst + v0) = make_float4(f[0], f[1], f[2], f[3]);
            }
        }
        // (released at once, the next kernel's CTAs pile up on the free SMs: 33 x 50021 fp32 3.2 against 4.6 us, 64 x 32000 2.5, 3.7)
        griddep_launch_dependents();
        // granules that the row only shares with its neighbours (a row inside one granule is a head)
        const bool head = f0 > 0, tail = f1 < row.count() && row.count() > f0;
        if (part == 0 && ((threadIdx.x == 0 && head) || (threadIdx.x == 1 && tail))) {
            const int32_t v0 = row.first(threadIdx.x == 0 ? 0 : row.count() - 1);
#pragma unroll 1
            for (int32_t v = max(v0, 0); v < v0 + E && v < p.V; ++v) from_float(r.grad(to_float(row.row[v]), v), dst[v]);
        }
    } else {
        const int64_t v1 = (int64_t)(part + 1) * p.span * E;
        for (int64_t v = (int64_t)part * p.span * E + threadIdx.x; v < v1 && v < p.V; v += GRAD_THREADS)
            from_float(r.grad(to_float(row.row[v]), v), dst[v]);
    }
}

template <typename T, int THREADS, int U, int STAGES, int RESIDENT, bool SELFTEST = false>
int launch_scores_cfg(const ScoreArgs &p, int cluster, cudaStream_t st)
{
    auto kern = scores_kernel<T, THREADS, U, STAGES, RESIDENT, SELFTEST>;
    constexpr size_t smem = sizeof(ScoreShared<THREADS, U, STAGES>);
    static_assert(smem * RESIDENT + 1024 * RESIDENT <= 228 * 1024, "shared memory of an SM");
    // the shared-memory opt-in is per kernel and device: asked for once each (racing first calls set the same attribute)
    static std::atomic<bool> done[64];
    int dev = 0;
    QNN_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
        QNN_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.T * cluster));
    cfg.blockDim = dim3(THREADS + 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    unsigned na = 0;
    if (cluster > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = (unsigned)cluster; attr[na].val.clusterDim.y = 1; attr[na].val.clusterDim.z = 1;
        ++na;
    }
    if (pdl_enabled()) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    cfg.attrs = attr; cfg.numAttrs = na;
    QNN_CUDA(cudaLaunchKernelEx(&cfg, kern, p));
    return check_launch("qnn_token_logprobs");
}

template <typename T>
int launch_scores(const ScoreArgs &p, cudaStream_t st)
{
    const int64_t granules = (int64_t)p.V / Granules<T>::E + 1;
    // CTAs a row.  128000 bf16 with 5 alternatives, 1 / 2 / 4 / 8 CTAs: 16 rows 13.6 / 10.0 / 7.6 / 6.9 us, 33 rows 14.0 / 10.1 / 8.1 /
    // 8.9, 64 rows 13.8 / 10.1 / 9.2 / 10.1, 74 rows 14.1 / 10.3 / 11.6 / 13.0, 100 rows 14.2 / 12.0 / 12.8 / 15.6, 296 rows 23.7 /
    // 21.3 / 27.7, 400 rows 26.8 / 30.1: two while they fit the SMs at four each, four at two each, eight at one each, less the
    // SMs that clusters of four and eight leave over.  And a part must be long enough to be worth a join, the more so the more
    // CTAs share an SM: 32000, 4 rows 6.1 / 5.4 / 5.1 / 5.5, 100 rows 7.0 / 6.8 / 7.5, 296 rows 8.5 / 9.3; 16384, 64 rows 5.6 / 5.2 / 6.1,
    // 100 rows 5.2 / 5.6; 50000, 200 rows 10.5 / 12.0.
    const int64_t sms = sm_count();
    int cluster = 1;
    for (int c = 2; c <= MAX_CLUSTER; c *= 2) {
        const int64_t ctas = p.T * c, least = ctas <= sms ? 768 : ctas <= 2 * sms ? 1536 : 6144;
        if (ctas * 10 <= sms * 8 / c * (c == 2 ? 10 : 9) && granules / c >= least) cluster = c;
    }
    // Threads a CTA: fewer a row, and so more rows on an SM, where rows are short and many -- the joins cost instructions in
    // every warp.  bf16, 8 alternatives, 64 / 128 / 256 threads: 592 x 2000 4.4 / 5.0 / 5.8 us, 4096 x 2000 13.6 / 20.1 / 33.4,
    // 296 x 4000 5.5 / 4.4 / 5.0, 296 x 8000 6.8 / 5.7 / 5.1, 444 x 8000 7.0 / 6.1 / 6.7, 4096 x 8000 27.4 / 28.4 / 40.8, 592 x 50000
    // 21.7 / 19.9 / 17.8, 1024 x 50000 33.7 / 28.4 / 29.5, 2048 x 131072 119 / 98 / 95.
    if (cluster > 1 || granules > 8192 || (granules > 640 && p.T <= 2 * sms) || (granules > 5000 && p.T <= 4 * sms))
        return launch_scores_cfg<T, 256, 4, 3, 4>(p, cluster, st);
    if (granules <= 320 || (granules <= 1024 && p.T > 7 * sms)) return launch_scores_cfg<T, 64, 4, 3, 12>(p, cluster, st);
    return launch_scores_cfg<T, 128, 4, 2, 8>(p, cluster, st);
}

template <typename T>
int launch_scores_grad(ScoreGradArgs p, int64_t rows, cudaStream_t st)
{
    constexpr int E = Granules<T>::E;
    const int64_t granules = (int64_t)p.V / E + 2;
    // Rounds a CTA: in 16 bits up to four while the SMs have eight CTAs each, to spread the set-up (2048 x 131072 bf16, kept up
    // for seconds: 165 against 173 us -- the power limit makes instructions count); in fp32 one (925 x 100544: 108 against 116).
    int64_t rounds = sizeof(T) == 4 ? 1 : rows * granules / ((int64_t)GRAD_THREADS * GRAD_U * 8 * sm_count());
    rounds = rounds < 1 ? 1 : rounds > 4 ? 4 : rounds;
    p.span = (int32_t)(GRAD_THREADS * GRAD_U * rounds);
    p.parts = (uint32_t)ceil_div(granules, p.span);
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
    QNN_REQUIRE(V <= ((int64_t)1 << 30) && T < ((int64_t)1 << 28), QNN_ERR_UNSUPPORTED, "%s: V above 2^30 or T of 2^28 and more", what);
    if (T == 0) return QNN_OK;
    QNN_REQUIRE(V >= 1, QNN_ERR_INVALID_ARG, "%s: V is 0", what);
    QNN_REQUIRE(logits != nullptr, QNN_ERR_INVALID_ARG, "%s: logits is NULL", what);
    QNN_REQUIRE(ldl >= V, QNN_ERR_INVALID_ARG, "%s: ldl below V", what);
    QNN_REQUIRE(aligned(logits, (size_t)type_bytes(type)), QNN_ERR_ALIGNMENT, "%s: logits are not aligned to their elements", what);
    return QNN_OK;
}

}  // namespace

int scores_selftest(uint8_t *scratch, cudaStream_t st)
{
    // one row of 16384 zeros, four CTAs, eight alternatives
    ScoreArgs p{};
    p.logits = scratch; p.T = 1; p.V = 16384; p.ldl = 16384; p.topk = 8;
    float *f = reinterpret_cast<float *>(scratch) + 16384;
    p.lse = f; p.entropy = f + 1; p.top_logprob = f + 2;
    static_assert((16384 + 2 + 8) * 4 <= CLUSTER_SELFTEST_BYTES, "scratch");
    return launch_scores_cfg<float, 256, 4, 3, 4, true>(p, 4, st);
}

int scores_status(int *code)
{
    QNN_CUDA(status_read_clear(code));
    return QNN_OK;
}

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
    p.logits = logits; p.T = T; p.ldl = ldl; p.V = (int32_t)V;
    p.ids = ids; p.logprob = logprob; p.entropy = entropy; p.lse = lse;
    p.topk = topk; p.top_logprob = top_logprob; p.top_ids = top_ids;
    cudaStream_t st = as_stream(stream);
    switch (type) {
        case QNN_TYPE_F32: return launch_scores<float>(p, st);
        case QNN_TYPE_BF16: return launch_scores<__nv_bfloat16>(p, st);
        default: return launch_scores<__half>(p, st);
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
