// int8 x int8 product with a scale for each token and each output channel:
//   out[m, n] = (float(sum_k a[m,k] b[n,k]) * a_scale[m]) * b_scale[n] + bias[n]
// The sum is exact in int32 (tcgen05 kind::i8 accumulates there), so it does not depend on tiles or splits.
//
// Three kernels:
//  - wide: persistent; tokens are the tile's 128 (a CTA pair: 256) rows, channels its columns.  Warp 0 loads by TMA, warp 1
//    multiplies into one of two accumulator stages in tensor memory, the other warps scale and store the previous tile.  Bound
//    by the tensor cores: 10000 x 4096 x 4096 in 110 to 113 us, 3000 T operations/s, their pipe busy 79 % of the time (nine waves of
//    tiles for 8.65; repeated for seconds the power limit holds it at 128 us).
//  - narrow, for few tokens: bound by the bytes of the weights and by latency, so weights are the tile's 128 rows and the tokens
//    its 16..128 columns; K is cut among the CTAs of a cluster, whose int32 partial sums meet in shared memory.  16 x 131072 x
//    4096: 88 us, 6.1 TB/s of weights; 100 x 4096 x 4096: 8.8 us, 7.6 where L2 still holds the weights.
//  - integer units, for one to four tokens: 1 x 4096 x 4096 in 5.2 us (3.2 TB/s of weights, launch and all), 2.9 where L2 still holds
//    them; 1 x 128000 x 4096 in 76 us (6.9 TB/s).
// All device-side waits are bounded.
#include <cuda.h>
#include <atomic>
#include "qnn_types.cuh"
#include "qnn_tc_ptx.cuh"

namespace qnn {
namespace {

struct I8sParams {
    int64_t M, N;
    int32_t num_kb;                  // K blocks of 128 bytes
    int32_t tiles_m, tiles_n;        // wide: in units of 128 * CTAS rows and BN columns
    const float *a_scale, *b_scale, *bias;
    void *out; int64_t ldo;
    int tma_out;                     // 1: bulk stores through tmap_out
    uint32_t idesc, idesc_last; int32_t n_last;   // the last column block multiplies n_last columns only
};

constexpr int tmem_cols(int c) { return c <= 32 ? 32 : c <= 64 ? 64 : c <= 128 ? 128 : c <= 256 ? 256 : 512; }

template <int BN, int CTAS, typename TOUT, int G>
struct WideCfg {
    static constexpr int THREADS = 64 + 128 * G;
    static constexpr int A_BYTES = BM * BKB;
    static constexpr int B_BYTES = (BN / CTAS) * BKB;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int CB = 128 / (int)sizeof(TOUT);                  // columns of a 128-byte staging row
    static constexpr int NB = BN / CB;                                  // staging blocks a tile
    static constexpr int NBW = (NB + G - 1) / G;                        // ... a warp
    static constexpr int STG_BYTES = 4 * G * 4096;
    static constexpr int COL_FLOATS = 2 * NBW * CB;                     // a warp's channel scales and biases
    static constexpr int COL_BYTES = 4 * G * COL_FLOATS * 4;
    static constexpr int AUX = 256 + COL_BYTES + 1024;
    static constexpr int MAXS = (SMEM_LIMIT - AUX - STG_BYTES) / STAGE_BYTES;
    static constexpr int STAGES = MAXS > 8 ? 8 : MAXS;
    static constexpr int STG_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int BAR_OFFSET = STG_OFFSET + STG_BYTES;
    static constexpr int COL_OFFSET = BAR_OFFSET + 256;
    static constexpr int TOTAL = COL_OFFSET + COL_BYTES + 1024;
    static constexpr int TMEM = tmem_cols(2 * BN);
    static_assert(STAGES >= 3 && TMEM <= 512 && BN % CB == 0 && (2 * STAGES + 4) * 8 + 8 <= 256, "configuration");
};

// 32 accumulator columns of one row -> scaled values; sb / bi: this block's channel scales and biases in shared memory
__device__ __forceinline__ void scale32(const uint32_t (&v)[32], float sa, const float *sb, const float *bi, float (&f)[32])
{
#pragma unroll
    for (int j4 = 0; j4 < 8; ++j4) {
        const float4 s = reinterpret_cast<const float4 *>(sb)[j4];      // the same address in every lane: a broadcast read
        const float4 b = reinterpret_cast<const float4 *>(bi)[j4];
        f[4 * j4] = fmaf(__int2float_rn((int32_t)v[4 * j4]) * sa, s.x, b.x);
        f[4 * j4 + 1] = fmaf(__int2float_rn((int32_t)v[4 * j4 + 1]) * sa, s.y, b.y);
        f[4 * j4 + 2] = fmaf(__int2float_rn((int32_t)v[4 * j4 + 2]) * sa, s.z, b.z);
        f[4 * j4 + 3] = fmaf(__int2float_rn((int32_t)v[4 * j4 + 3]) * sa, s.w, b.w);
    }
}

template <int BN, int CTAS, typename TOUT, int G>
__global__ void __launch_bounds__(64 + 128 * G, 1)
gemm_i8s_wide_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                     const __grid_constant__ CUtensorMap tmap_out, const I8sParams p)
{
    using S = WideCfg<BN, CTAS, TOUT, G>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                      // swizzled tiles need 1024-byte alignment
    uint8_t *gen = smem_raw + (base - raw);
    const uint32_t bar0 = base + S::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(S::STAGES + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + 2 + a); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gen + S::BAR_OFFSET + 8 * (2 * S::STAGES + 4));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    // a pair's CTA 0 leads: it owns the full and accumulator-empty barriers and issues the products
    const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 4 * G * CTAS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<CTAS>(smem_u32(tmem_slot), S::TMEM);
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();                                 // the peer's barriers exist before anything arrives on them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // only now may the next kernel be scheduled: one that shares this SM could take the tensor memory this CTA waits for
    griddep_launch_dependents();
    griddep_wait();

    const uint32_t tiles_m = (uint32_t)p.tiles_m;
    const uint32_t num_tiles = tiles_m * (uint32_t)p.tiles_n;          // below 2^31 (checked on the host)
    const uint32_t step_n = (gridDim.x / CTAS) / tiles_m, step_m = (gridDim.x / CTAS) - step_n * tiles_m;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0;
            bool ok = true, ready = false;
            const uint32_t tx_bytes = (uint32_t)S::STAGE_BYTES * CTAS;
            const uint32_t fb0 = (CTAS == 2) ? map_to_cta(full_bar(0), 0) : full_bar(0), eb0 = empty_bar(0);
            uint32_t sa = base, fb = fb0, eb = eb0;
            int32_t tn = (int32_t)((blockIdx.x / CTAS) / tiles_m), tm = (int32_t)((blockIdx.x / CTAS) - (uint32_t)tn * tiles_m);
            for (uint32_t t = blockIdx.x / CTAS; t < num_tiles && ok; t += gridDim.x / CTAS) {
                const int32_t a_row = (CTAS == 2) ? (tm * 2 + (int32_t)rank) * BM : tm * BM;
                const int32_t b_row = (CTAS == 2) ? tn * BN + (int32_t)rank * ((tn == p.tiles_n - 1 ? p.n_last : BN) / 2) : tn * BN;
                int32_t kx = 0;
#pragma unroll 1
                for (int32_t kb = 0; kb < p.num_kb; ++kb) {
                    if (!ready && !mbar_wait(eb, phase ^ 1u, abort_flag, 11)) { ok = false; break; }
                    const bool wrap = stage == S::STAGES - 1;
                    const uint32_t sa_n = wrap ? base : sa + (uint32_t)S::STAGE_BYTES;
                    const uint32_t fb_n = wrap ? fb0 : fb + 8u;
                    const uint32_t eb_n = wrap ? eb0 : eb + 8u;
                    const uint32_t phase_n = wrap ? phase ^ 1u : phase;
                    if (CTAS == 2)
                        ready = tma_stage_2d_pair(eb_n, phase_n ^ 1u, fb, tx_bytes, (uint32_t)leader, sa, &tmap_a, kx, a_row, sa + S::A_BYTES,
                                                  &tmap_b, kx, b_row) != 0;
                    else
                        ready = tma_stage_2d(eb_n, phase_n ^ 1u, fb, tx_bytes, sa, &tmap_a, kx, a_row, sa + S::A_BYTES, &tmap_b, kx, b_row) != 0;
                    kx += BKB;
                    stage = wrap ? 0 : stage + 1;
                    sa = sa_n; fb = fb_n; eb = eb_n; phase = phase_n;
                }
                tm += (int32_t)step_m; tn += (int32_t)step_n;
                if (tm >= (int32_t)tiles_m) { tm -= (int32_t)tiles_m; ++tn; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            int stage = 0; uint32_t phase = 0, iter = 0;
            bool ok = true, ready = false;
            const uint64_t desc0 = make_kmajor_desc<BKB>(base);
            const uint32_t desc_hi = (uint32_t)(desc0 >> 32);
            const uint32_t a_lo0 = (uint32_t)desc0, fb0 = full_bar(0), eb0 = empty_bar(0);
            uint32_t a_lo = a_lo0, fb = fb0, eb = eb0;
            uint32_t tn = (blockIdx.x / CTAS) / tiles_m, tm = (blockIdx.x / CTAS) - tn * tiles_m;
            for (uint32_t t = blockIdx.x / CTAS; t < num_tiles && ok; t += gridDim.x / CTAS, ++iter) {
                const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
                const uint32_t idesc = (tn == (uint32_t)p.tiles_n - 1u) ? p.idesc_last : p.idesc;
                tm += step_m; tn += step_n;
                if (tm >= tiles_m) { tm -= tiles_m; ++tn; }
                if (!mbar_wait(tempty_bar(as), aphase ^ 1u, abort_flag, 12)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + as * (uint32_t)BN;
#pragma unroll 4
                for (int32_t kb = 0; kb < p.num_kb; ++kb) {
                    if (!ready && !mbar_wait(fb, phase, abort_flag, 13)) { ok = false; break; }
                    const bool wrap = stage == S::STAGES - 1;
                    const uint32_t a_lo_n = wrap ? a_lo0 : a_lo + (uint32_t)(S::STAGE_BYTES >> 4);
                    const uint32_t fb_n = wrap ? fb0 : fb + 8u;
                    const uint32_t eb_n = wrap ? eb0 : eb + 8u;
                    const uint32_t phase_n = wrap ? phase ^ 1u : phase;
                    const uint32_t b_lo = a_lo + (uint32_t)(S::A_BYTES >> 4);
                    if (CTAS == 2)
                        ready = umma_stage_pair<QNN_FORM_I8>(fb_n, phase_n, d_tmem, a_lo, b_lo, desc_hi, idesc, (uint32_t)(kb != 0), 0u, eb) != 0;
                    else
                        ready = umma_stage<QNN_FORM_I8>(fb_n, phase_n, d_tmem, a_lo, b_lo, desc_hi, idesc, (uint32_t)(kb != 0), 0u, eb) != 0;
                    stage = wrap ? 0 : stage + 1;
                    a_lo = a_lo_n; fb = fb_n; eb = eb_n; phase = phase_n;
                }
                if (ok) {                                        // accumulator complete
                    if (CTAS == 2) umma_commit_pair(tfull_bar(as));
                    else umma_commit(tfull_bar(as));
                }
            }
        }
    } else {
        const int q = warp & 3;                                  // tensor-memory lane quarter this warp may read
        const int grp = (warp - 2) >> 2;
        const int ew = grp * 4 + q;
        float *cs = reinterpret_cast<float *>(gen + S::COL_OFFSET) + ew * S::COL_FLOATS;     // this warp's channel scales
        float *cb = cs + S::NBW * S::CB;                                                     // and biases
        uint8_t *stg = gen + S::STG_OFFSET + ew * 4096;
        const uint32_t stg_u32 = base + (uint32_t)(S::STG_OFFSET + ew * 4096);
        uint32_t iter = 0;
        bool ok = true;
        int32_t tn = (int32_t)((blockIdx.x / CTAS) / tiles_m), tm = (int32_t)((blockIdx.x / CTAS) - (uint32_t)tn * tiles_m);
        // Channel scales, biases and the token's scale of a tile are fetched into registers while the tile before it is
        // drained, and parked in shared memory when its turn comes: their latency never sits between two tiles.
        constexpr int CPL = S::NBW * S::CB / 32;                 // channels a lane fetches
        float s_next[CPL], b_next[CPL], sa_next;
        auto fetch = [&](int32_t ftm, int32_t ftn) {
            const int64_t m = ((int64_t)ftm * CTAS + rank) * BM + q * 32 + lane;
            sa_next = m < p.M ? __ldg(p.a_scale + m) : 0.0f;
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
                const int blk = grp + (i * 32 / S::CB) * G;
                const int64_t n = (int64_t)ftn * BN + blk * S::CB + (i * 32) % S::CB + lane;
                const bool in = blk < S::NB && n < p.N;
                s_next[i] = in ? __ldg(p.b_scale + n) : 0.0f;
                b_next[i] = in && p.bias ? __ldg(p.bias + n) : 0.0f;
            }
        };
        if (blockIdx.x / CTAS < num_tiles) fetch(tm, tn);
        for (uint32_t t = blockIdx.x / CTAS; t < num_tiles && ok; t += gridDim.x / CTAS, ++iter) {
            const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
            const int64_t ntile = (int64_t)tn * BN;
            const int64_t m0 = ((int64_t)tm * CTAS + rank) * BM + q * 32;       // the row of the warp's lane 0
            const float sa = sa_next;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
                cs[i * 32 + lane] = s_next[i];
                cb[i * 32 + lane] = b_next[i];
            }
            __syncwarp();
            tm += (int32_t)step_m; tn += (int32_t)step_n;        // the next tile's coordinates
            if (tm >= (int32_t)tiles_m) { tm -= (int32_t)tiles_m; ++tn; }
            if (t + gridDim.x / CTAS < num_tiles) fetch(tm, tn);
            // the tensor-memory loads below are warp-collective: leave the loop only as a whole warp
            if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(as), aphase, abort_flag, 14))) { ok = false; break; }
            tc_fence_after();
            const uint32_t tacc = tmem_base + ((uint32_t)(q * 32) << 16) + as * (uint32_t)BN;
            int nblk = (int)((p.N - ntile + S::CB - 1) / S::CB);
            nblk = nblk > S::NB ? S::NB : nblk;
            if (m0 >= p.M) nblk = 0;                             // (warp-uniform)
#pragma unroll 1
            for (int blk = grp, b = 0; blk < nblk; blk += G, ++b) {
                const int64_t n0 = ntile + blk * S::CB;
                if (lane == 0) bulk_wait_read<0>();              // this warp's previous store has read the tile
                __syncwarp();
#pragma unroll
                for (int h = 0; h < S::CB / 32; ++h) {
                    uint32_t v[32];
                    float f[32];
                    tmem_ld32(tacc + (uint32_t)(blk * S::CB + h * 32), v);
                    scale32(v, sa, cs + b * S::CB + h * 32, cb + b * S::CB + h * 32, f);
                    // row `lane` of the staging tile, 16-byte chunks swizzled by the row (the tensor map's 128-byte swizzle)
                    if constexpr (sizeof(TOUT) == 4) {
#pragma unroll
                        for (int ch = 0; ch < 8; ++ch)
                            *reinterpret_cast<float4 *>(stg + lane * 128 + ((ch ^ (lane & 7)) << 4)) =
                                make_float4(f[4 * ch], f[4 * ch + 1], f[4 * ch + 2], f[4 * ch + 3]);
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            *reinterpret_cast<uint4 *>(stg + lane * 128 + (((h * 4 + c) ^ (lane & 7)) << 4)) =
                                make_uint4(pack2(f[8 * c], f[8 * c + 1], TOUT()), pack2(f[8 * c + 2], f[8 * c + 3], TOUT()),
                                           pack2(f[8 * c + 4], f[8 * c + 5], TOUT()), pack2(f[8 * c + 6], f[8 * c + 7], TOUT()));
                    }
                }
                if (p.tma_out) {
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&tmap_out, (int32_t)n0, (int32_t)m0, stg_u32);
                        bulk_commit();
                    }
                } else {
                    // rows of any alignment: lanes along the columns, element by element
                    __syncwarp();
                    const int rows = p.M - m0 < 32 ? (int)(p.M - m0) : 32;
                    TOUT *dst = static_cast<TOUT *>(p.out) + m0 * p.ldo + n0 + lane;
#pragma unroll (sizeof(TOUT) == 4 ? 8 : 4)
                    for (int r = 0; r < rows; ++r, dst += p.ldo) {
#pragma unroll
                        for (int h = 0; h < S::CB / 32; ++h) {
                            const int byte = (h * 32 + lane) * (int)sizeof(TOUT);
                            const TOUT x = *reinterpret_cast<const TOUT *>(stg + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15));
                            if (n0 + h * 32 + lane < p.N) dst[h * 32] = x;
                        }
                    }
                    __syncwarp();
                }
            }
            // all reads of this accumulator stage are done: hand it back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CTAS == 2) mbar_arrive_cluster(map_to_cta(tempty_bar(as), 0));
                else mbar_arrive(tempty_bar(as));
            }
        }
        if (lane == 0) bulk_wait_all();                          // stores must have read shared memory before it goes away
        __syncwarp();
    }

    __syncwarp();
    if (*abort_flag) let_flights_land();
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();     // the peer no longer touches this CTA's barriers, shared or tensor memory
    tc_fence_after();
    if (warp == 1) tmem_dealloc<CTAS>(tmem_base, S::TMEM);
}

// ---- few tokens ------------------------------------------------------------------------------------------------

constexpr int NARROW_THREADS = 192;        // warp 0: TMA, warp 1: products, warps 2..5: sums and stores

template <int BN>
struct NarrowCfg {
    static constexpr int A_BYTES = BM * BKB;                            // weights
    static constexpr int B_BYTES = BN * BKB;                            // tokens
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    // How the partial sums of a cluster meet.  Up to 16 tokens every thread sends its few to the CTA that joins them, which
    // waits on a barrier of its own: no cluster-wide barrier after the products (16 x 4096 x 4096: half a microsecond less).  With
    // more tokens the stores are too many (100 tokens: 1.7 us slower): sums go to shared memory, over the operand stages, and
    // are read from there in 16-byte pieces; so they are where K is not cut, to be stored along the channels (100 x 16384 x
    // 4096: 16.6 us, by thread and column 19.9).
    static constexpr bool PUSH = BN == 16;
    // Up to 64 tokens two CTAs fit an SM: one's set-up and join overlap the other's stream of weights.  With 128 a stage is so
    // large that two CTAs would have three each, too little in flight: one CTA with six (100 x 4096 x 4096: 7.7 us against 8.7 us,
    // 128 x 16384 x 4096 19.9 against 24.5).
    static constexpr int RESIDENT = BN == 128 ? 1 : 2;
    static constexpr int STAGES = BN == 128 ? 6 : BN == 16 ? 5 : (108 * 1024) / STAGE_BYTES > 6 ? 6 : (108 * 1024) / STAGE_BYTES;
    static constexpr int JOIN_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int BAR_OFFSET = JOIN_OFFSET + (PUSH ? BM * BN * 4 : 0);
    static constexpr int SCALE_OFFSET = BAR_OFFSET + 128;               // the tokens' scales
    static constexpr int TOTAL = SCALE_OFFSET + BN * 4 + 1024;
    static constexpr int TMEM = tmem_cols(BN);
    static_assert(PUSH || STAGES * STAGE_BYTES >= BN * BM * 4, "the partial sums reuse the stages");
    static_assert((2 * STAGES + 2) * 8 + 8 <= 128 && RESIDENT * (TOTAL + 1024) <= 228 * 1024, "configuration");
};

__device__ __forceinline__ int4 ld_peer_i32x4(uint32_t addr)
{
    int4 v;
    asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// asynchronous store of W int32 into another CTA's shared memory that reports its bytes to a barrier there
template <int W>
__device__ __forceinline__ void send_i32(uint32_t addr, const uint32_t *v, uint32_t bar)
{
    if constexpr (W == 4)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                     ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(bar) : "memory");
    else
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];"
                     ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// SELFTEST: CTA 1 of a cluster gives up before it sends, CTA 2 sends late, and the others wait for a short time only.
template <int BN, typename TOUT, int SPLIT, bool SELFTEST = false>
__global__ void __launch_bounds__(NARROW_THREADS, NarrowCfg<BN>::RESIDENT)
gemm_i8s_narrow_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const I8sParams p)
{
    using S = NarrowCfg<BN>;
    constexpr int split = SPLIT;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *gen = smem_raw + (base - raw);
    const uint32_t bar0 = base + S::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(S::STAGES + s); };
    const uint32_t done_bar = bar0 + 8u * (uint32_t)(2 * S::STAGES);
    const uint32_t join_bar = done_bar + 8u;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gen + S::BAR_OFFSET + 8 * (2 * S::STAGES + 2));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    float *token_scale = reinterpret_cast<float *>(gen + S::SCALE_OFFSET);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x % (uint32_t)split;                // = the CTA's rank in its cluster
    const uint32_t tile = blockIdx.x / (uint32_t)split;
    const int32_t tn = (int32_t)(tile % (uint32_t)p.tiles_n), tm = (int32_t)(tile / (uint32_t)p.tiles_n);
    const int32_t kb0 = (int32_t)((int64_t)p.num_kb * rank / split), kb1 = (int32_t)((int64_t)p.num_kb * (rank + 1) / split);
    const int32_t nt = p.M - (int64_t)tm * BN < BN ? (int32_t)(p.M - (int64_t)tm * BN) : BN;   // tokens of this tile
    // (PUSH) CTA r of a cluster joins tokens r * TPO .. r * TPO + TPO - 1, W of them to a store
    constexpr int TPO = BN / SPLIT, W = TPO < 4 ? TPO : 4;
    const int32_t own = nt - (int32_t)rank * TPO;                      // ... of which it has this many
    const int32_t own_groups = own <= 0 ? 0 : own >= TPO ? TPO / W : (own + W - 1) / W;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        mbar_init(done_bar, 1);
        mbar_init(join_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        // what the CTAs of the cluster send here
        if (S::PUSH && SPLIT > 1)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(join_bar), "r"((uint32_t)(SPLIT * BM * own_groups * W * 4)) : "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_u32(tmem_slot), S::TMEM);
    if (warp == 2 && lane < 2)
        asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &tmap_w : &tmap_x) : "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (S::PUSH && SPLIT > 1) cluster_arrive();                        // nothing is sent before every CTA's barrier stands
    // When the next kernel may be scheduled (after the allocation, as above): at once where it cannot share an SM with this one;
    // else when the last loads are on their way -- earlier its CTAs pile up, two to an SM, on the SMs that are free and stay
    // there (64 x 4096 x 4096 6.5 against 7.4 us, 16 x 4096 x 4096 4.9 against 5.2).
    if (S::RESIDENT == 1) griddep_launch_dependents();
    griddep_wait();

    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0;
            for (int32_t kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, 15)) break;
                const uint32_t sa = base + (uint32_t)(stage * S::STAGE_BYTES);
                (void)tma_stage_2d(empty_bar(stage), phase ^ 1u, full_bar(stage), (uint32_t)S::STAGE_BYTES, sa, &tmap_w, kb * BKB, tn * BM,
                                   sa + S::A_BYTES, &tmap_x, kb * BKB, tm * BN);
                if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
            }
            if (S::RESIDENT > 1) griddep_launch_dependents();
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0;
            const uint64_t desc0 = make_kmajor_desc<BKB>(base);
            const uint32_t desc_hi = (uint32_t)(desc0 >> 32);
            bool fine = true;
            for (int32_t kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait(full_bar(stage), phase, abort_flag, 16)) { fine = false; break; }
                const uint32_t a_lo = (uint32_t)desc0 + (uint32_t)(stage * (S::STAGE_BYTES >> 4));
                (void)umma_stage<QNN_FORM_I8>(full_bar(stage), phase, tmem_base, a_lo, a_lo + (uint32_t)(S::A_BYTES >> 4), desc_hi, p.idesc,
                                              (uint32_t)(kb != kb0), 0u, empty_bar(stage));
                if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
            }
            if (fine) umma_commit(done_bar);
        }
    } else {
        const int q = warp & 3;
        const int n_local = q * 32 + lane;
        const int64_t n = (int64_t)tn * BM + n_local;
        // the scales are fetched while the products run
        if (n_local < nt) token_scale[n_local] = __ldg(p.a_scale + (int64_t)tm * BN + n_local);
        float sb = 0.0f, bi = 0.0f;
        if (S::PUSH) {
            if (n < p.N) sb = __ldg(p.b_scale + n);
            if (n < p.N && p.bias) bi = __ldg(p.bias + n);
            asm volatile("barrier.sync 1, 128;" ::: "memory");
        }
        ok = __all_sync(0xffffffffu, mbar_wait(done_bar, 0, abort_flag, 17));
        if (S::PUSH && SPLIT > 1) cluster_wait();
        if (SELFTEST && rank == 1) { *abort_flag = 1; ok = false; }
        if (SELFTEST && rank == 2)
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        if (ok) {
            tc_fence_after();
            auto store = [&](int j, int32_t sum) {               // token j of the tile, this thread's channel
                const int64_t m = (int64_t)tm * BN + j;
                if (n < p.N) from_float(fmaf(__int2float_rn(sum) * token_scale[j], sb, bi), static_cast<TOUT *>(p.out)[m * p.ldo + n]);
            };
            int32_t *dump = reinterpret_cast<int32_t *>(gen);    // (not PUSH) [token][128 channels], over the operand stages
#pragma unroll 1
            for (int c = 0; c < nt; c += 16) {
                uint32_t v[16];
                tmem_ld16(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)c, v);
                if constexpr (!S::PUSH) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < nt) dump[(c + j) * BM + n_local] = (int32_t)v[j];
                } else if (SPLIT == 1) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < nt) store(c + j, (int32_t)v[j]);
                } else {
                    // W tokens of this channel to the CTA that joins them: [sender][group of W tokens][channel][W]
#pragma unroll
                    for (int g = 0; g < 16; g += W) {
                        const int j = c + g, owner = j / TPO;
                        if (j < nt)
                            send_i32<W>(map_to_cta(base + (uint32_t)(S::JOIN_OFFSET + (((int)rank * (TPO / W) + (j - owner * TPO) / W) * BM + n_local) * W * 4), (uint32_t)owner),
                                        v + g, map_to_cta(join_bar, (uint32_t)owner));
                    }
                }
            }
            if (S::PUSH && SPLIT > 1 && own_groups > 0) {
                ok = __all_sync(0xffffffffu, mbar_wait(join_bar, 0, abort_flag, 18, SELFTEST ? 64u : WAIT_LIMIT));
                const int32_t *part = reinterpret_cast<const int32_t *>(gen + S::JOIN_OFFSET) + n_local * W;
                for (int g = 0; g < own_groups && ok; ++g) {
                    int32_t sum[W];
#pragma unroll
                    for (int i = 0; i < W; ++i) sum[i] = 0;
#pragma unroll
                    for (int r = 0; r < SPLIT; ++r) {
                        alignas(16) int32_t x[W];
                        if constexpr (W == 4) *reinterpret_cast<int4 *>(x) = *reinterpret_cast<const int4 *>(part + (r * (TPO / W) + g) * BM * W);
                        else *reinterpret_cast<int2 *>(x) = *reinterpret_cast<const int2 *>(part + (r * (TPO / W) + g) * BM * W);
#pragma unroll
                        for (int i = 0; i < W; ++i) sum[i] += x[i];
                    }
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const int j = (int)rank * TPO + g * W + i;
                        if (j < nt) store(j, sum[i]);
                    }
                }
            }
        }
    }
    __syncwarp();
    if (S::PUSH && SPLIT > 1 && warp < 2) cluster_wait();               // (as the other warps did above)
    if (!S::PUSH) {
        // A warp takes a few tokens at a time, a lane four channels of them: 16 16-byte reads from the CTAs of the cluster are on
        // their way before the first is used.
        const int64_t n = (int64_t)tn * BM + 4 * lane;
        float sb[4], bi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sb[i] = n + i < p.N ? __ldg(p.b_scale + n + i) : 0.0f;
            bi[i] = n + i < p.N && p.bias ? __ldg(p.bias + n + i) : 0.0f;
        }
        // every CTA of the cluster reaches both barriers, whatever became of its waits
        if (SPLIT > 1) cluster_sync_all();
        else __syncthreads();
        constexpr int AT_ONCE = 16 / SPLIT, STRIDE = SPLIT * (NARROW_THREADS / 32);
#pragma unroll 1
        for (int j0 = (int)rank + warp * SPLIT; j0 < nt; j0 += AT_ONCE * STRIDE) {
            int4 v[AT_ONCE][SPLIT];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                for (int r = 0; r < SPLIT; ++r)
                    if (j0 + i * STRIDE < nt)
                        v[i][r] = ld_peer_i32x4(map_to_cta(base + (uint32_t)(((j0 + i * STRIDE) * BM + 4 * lane) * 4), (uint32_t)r));
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int j = j0 + i * STRIDE;
                if (j >= nt) break;
                const int64_t m = (int64_t)tm * BN + j;
                const float sa = token_scale[j];
                int4 s = v[i][0];
#pragma unroll
                for (int r = 1; r < SPLIT; ++r) { s.x += v[i][r].x; s.y += v[i][r].y; s.z += v[i][r].z; s.w += v[i][r].w; }
                const float f[4] = {fmaf(__int2float_rn(s.x) * sa, sb[0], bi[0]), fmaf(__int2float_rn(s.y) * sa, sb[1], bi[1]),
                                    fmaf(__int2float_rn(s.z) * sa, sb[2], bi[2]), fmaf(__int2float_rn(s.w) * sa, sb[3], bi[3])};
                TOUT *dst = static_cast<TOUT *>(p.out) + m * p.ldo + n;
                if (n + 4 <= p.N && (reinterpret_cast<uintptr_t>(dst) & (4 * sizeof(TOUT) - 1)) == 0) {
                    if constexpr (sizeof(TOUT) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(f[0], f[1], f[2], f[3]);
                    else *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2(f[0], f[1], TOUT()), pack2(f[2], f[3], TOUT()));
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (n + k < p.N) from_float(f[k], dst[k]);
                }
            }
        }
        if (SPLIT > 1) cluster_sync_all();                // nobody leaves while its partial sums are being read
    }
    tc_fence_before();
    const bool aborted = __syncthreads_or(*abort_flag) != 0;
    tc_fence_after();
    if (aborted) {
        // (PUSH) the CTAs of the cluster may not have sent everything yet
        if (S::PUSH && SPLIT > 1) stay_for_cluster();
        else let_flights_land();
    }
    if (warp == 1) tmem_dealloc<1>(tmem_base, S::TMEM);
}

// ---- a handful of tokens ---------------------------------------------------------------------------------------
//
// Bound by reading the weights once, and at 2.6 us of it (16.8 MB at the copy rate) by latency: a launch, one round of loads, a sum.  So no
// shared-memory staging and no tensor memory: a warp reads GEMV_R rows of weights 16 bytes a lane, multiplies by the tokens'
// codes (which stay in L1) four at a time on the integer units (dp4a), and sums over its lanes.  K may be cut among the warps
// of a block, whose partial sums meet in shared memory.

__device__ __forceinline__ uint4 load_codes(const uint8_t *row, int32_t k) { return __ldg(reinterpret_cast<const uint4 *>(row + k)); }
// the same with the codes from K on taken as 0 (only one factor of a product needs it)
__device__ __forceinline__ uint4 load_codes_to(const uint8_t *row, int32_t k, int32_t K)
{
    uint4 v = load_codes(row, k);
    const int left = K - k;                                  // >= 1
    if (left < 16) {
        auto keep = [&](int first) { const int n = left - first; return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; };
        v.x &= keep(0); v.y &= keep(4); v.z &= keep(8); v.w &= keep(12);
    }
    return v;
}
__device__ __forceinline__ int32_t dot16(const uint4 &a, const uint4 &b, int32_t s)
{
    s = __dp4a((int)a.x, (int)b.x, s);
    s = __dp4a((int)a.y, (int)b.y, s);
    s = __dp4a((int)a.z, (int)b.z, s);
    return __dp4a((int)a.w, (int)b.w, s);
}

template <int MT, int GEMV_R, int GEMV_U, typename TOUT>
__global__ void __launch_bounds__(256) gemv_i8s_kernel(const uint8_t *__restrict__ a, int64_t lda, const uint8_t *__restrict__ b, int64_t ldb,
                                                       const int32_t K, const int ksplit, const I8sParams p)
{
    __shared__ int32_t part[8][GEMV_R * MT];
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per_block = 8 / ksplit;                        // row groups of a block
    const int64_t n0 = ((int64_t)blockIdx.x * per_block + warp / ksplit) * GEMV_R;
    const int32_t share = (((K + 15) / 16 + ksplit - 1) / ksplit) * 16;    // codes of a warp's part of K
    const int32_t k0 = share * (warp % ksplit), k1 = k0 + share < K ? k0 + share : K;
    int32_t acc[GEMV_R][MT];
#pragma unroll
    for (int r = 0; r < GEMV_R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[r][m] = 0;
    const uint8_t *br[GEMV_R], *ar[MT];
#pragma unroll
    for (int r = 0; r < GEMV_R; ++r) br[r] = b + (n0 + r < p.N ? n0 + r : p.N - 1) * ldb;
#pragma unroll
    for (int m = 0; m < MT; ++m) ar[m] = a + (m < p.M ? m : p.M - 1) * lda;
    int32_t k = k0 + 16 * lane;
    // whole rounds: GEMV_U x GEMV_R loads of weights in flight
    for (; k + 512 * (GEMV_U - 1) + 16 <= k1; k += 512 * GEMV_U) {
        uint4 w[GEMV_U][GEMV_R];
#pragma unroll
        for (int u = 0; u < GEMV_U; ++u)
#pragma unroll
            for (int r = 0; r < GEMV_R; ++r) w[u][r] = load_codes(br[r], k + 512 * u);
#pragma unroll
        for (int u = 0; u < GEMV_U; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint4 x = load_codes(ar[m], k + 512 * u);
#pragma unroll
                for (int r = 0; r < GEMV_R; ++r) acc[r][m] = dot16(w[u][r], x, acc[r][m]);
            }
    }
    for (; k < k1; k += 512) {
        uint4 w[GEMV_R];
#pragma unroll
        for (int r = 0; r < GEMV_R; ++r) w[r] = load_codes(br[r], k);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const uint4 x = load_codes_to(ar[m], k, K);
#pragma unroll
            for (int r = 0; r < GEMV_R; ++r) acc[r][m] = dot16(w[r], x, acc[r][m]);
        }
    }
    // the weights are in: the next kernel may be scheduled now (allowed to start at once, its blocks pile up on the SMs that are
    // free, several to one, and stay there: 1 x 4096 x 4096 2.8 against 3.4 us)
    griddep_launch_dependents();
    int32_t mine = 0;                                        // lane r * MT + m keeps sum (r, m)
#pragma unroll
    for (int r = 0; r < GEMV_R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int32_t s = __reduce_add_sync(0xffffffffu, acc[r][m]);
            if (lane == r * MT + m) mine = s;
        }
    if (ksplit > 1) {
        if (lane < GEMV_R * MT) part[warp][lane] = mine;
        __syncthreads();
        if (warp % ksplit != 0) return;
        if (lane < GEMV_R * MT)
            for (int i = 1; i < ksplit; ++i) mine += part[warp + i][lane];
    }
    const int64_t n = n0 + lane / MT;
    const int m = lane % MT;
    if (lane < GEMV_R * MT && n < p.N && m < p.M) {
        const float f = fmaf(__int2float_rn(mine) * __ldg(p.a_scale + m), __ldg(p.b_scale + n), p.bias ? __ldg(p.bias + n) : 0.0f);
        from_float(f, static_cast<TOUT *>(p.out)[m * p.ldo + n]);
    }
}

// K = 0: the bias alone
template <typename TOUT>
__global__ void __launch_bounds__(256) bias_rows_kernel(int64_t M, int64_t N, const float *__restrict__ bias, TOUT *__restrict__ out, int64_t ldo)
{
    griddep_launch_dependents();
    griddep_wait();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < M * N; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t m = i / N, n = i - m * N;
        from_float(bias ? bias[n] : 0.0f, out[m * ldo + n]);
    }
}

int make_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, int64_t rows, int64_t cols, int64_t ld_bytes, int box_rows,
             int box_cols, CUtensorMapL2promotion promo)
{
    EncodeTiledFn fn = encode_fn();
    QNN_REQUIRE(fn != nullptr, QNN_ERR_CUDA, "qnn_gemm_i8_scaled: cuTensorMapEncodeTiled is not available from this driver");
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld_bytes};
    cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = fn(map, type, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    promo, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    QNN_REQUIRE(r == CUDA_SUCCESS, QNN_ERR_CUDA, "qnn_gemm_i8_scaled: cuTensorMapEncodeTiled failed with code %d", (int)r);
    return QNN_OK;
}
int make_map_codes(CUtensorMap *map, const void *base, int64_t rows, int64_t K, int64_t ld, int box_rows)
{
    return make_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, rows, K, ld, box_rows, BKB, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

constexpr uint32_t i8_idesc(int m, int n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// The shared-memory opt-in is per kernel and device and costs microseconds: asked for once each.  (Racing first calls of two
// host threads set the same attribute, which is harmless.)
template <typename Kern>
int opt_in(Kern kern, int bytes, std::atomic<bool> (&done)[64])
{
    int dev = 0;
    QNN_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
        QNN_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
    }
    return QNN_OK;
}

template <class... KArgs, class... Args>
cudaError_t launch_clustered(void (*kernel)(KArgs...), unsigned grid, unsigned block, size_t smem, int cluster, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
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
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

struct I8sCall {
    const void *a, *b;
    int64_t lda, ldb, K;
};

template <int BN, typename TOUT, int SPLIT, bool SELFTEST = false>
int launch_narrow_split(const I8sCall &c, I8sParams p, cudaStream_t st)
{
    using S = NarrowCfg<BN>;
    auto kern = gemm_i8s_narrow_kernel<BN, TOUT, SPLIT, SELFTEST>;
    static std::atomic<bool> done[64];
    if (int rc = opt_in(kern, S::TOTAL, done)) return rc;
    CUtensorMap mw, mx;
    if (int rc = make_map_codes(&mw, c.b, p.N, c.K, c.ldb, BM)) return rc;
    if (int rc = make_map_codes(&mx, c.a, p.M, c.K, c.lda, BN)) return rc;
    p.idesc = i8_idesc(BM, BN);
    const int64_t ctas = (int64_t)p.tiles_n * p.tiles_m * SPLIT;
    QNN_REQUIRE(ctas < ((int64_t)1 << 31), QNN_ERR_UNSUPPORTED, "qnn_gemm_i8_scaled: too many output tiles");
    profile_before(st);
    QNN_CUDA(launch_clustered(kern, (unsigned)ctas, NARROW_THREADS, S::TOTAL, SPLIT, st, mw, mx, p));
    profile_after(st);
    return check_launch("qnn_gemm_i8_scaled");
}
template <int BN, typename TOUT>
int launch_narrow(const I8sCall &c, I8sParams p, int split, cudaStream_t st)
{
    p.tiles_n = (int32_t)ceil_div(p.N, BM);
    p.tiles_m = (int32_t)ceil_div(p.M, BN);
    switch (split) {
        case 1: return launch_narrow_split<BN, TOUT, 1>(c, p, st);
        case 2: return launch_narrow_split<BN, TOUT, 2>(c, p, st);
        case 4: return launch_narrow_split<BN, TOUT, 4>(c, p, st);
        default: return launch_narrow_split<BN, TOUT, 8>(c, p, st);
    }
}

template <int BN, int CTAS, typename TOUT>
int launch_wide(const I8sCall &c, I8sParams p, int workers, cudaStream_t st)
{
    constexpr int G = 2;
    using S = WideCfg<BN, CTAS, TOUT, G>;
    auto kern = gemm_i8s_wide_kernel<BN, CTAS, TOUT, G>;
    static std::atomic<bool> done[64];
    if (int rc = opt_in(kern, S::TOTAL, done)) return rc;
    CUtensorMap ma, mb, mo;
    if (int rc = make_map_codes(&ma, c.a, p.M, c.K, c.lda, BM)) return rc;
    if (int rc = make_map_codes(&mb, c.b, p.N, c.K, c.ldb, BN / CTAS)) return rc;
    mo = ma;
    // the bulk store clips the rows' extent in 16-byte units
    p.tma_out = aligned(p.out, 16) && (p.ldo * sizeof(TOUT)) % 16 == 0 && (p.N * sizeof(TOUT)) % 16 == 0;
    if (p.tma_out) {
        const CUtensorMapDataType dt = sizeof(TOUT) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
        if (int rc = make_map(&mo, dt, p.out, p.M, p.N, p.ldo * (int64_t)sizeof(TOUT), 32, S::CB, CU_TENSOR_MAP_L2_PROMOTION_NONE))
            return rc;
    }
    p.tiles_n = (int32_t)ceil_div(p.N, BN);
    p.tiles_m = (int32_t)ceil_div(p.M, BM * CTAS);
    const int64_t rest = p.N - (int64_t)(p.tiles_n - 1) * BN;
    p.n_last = (int32_t)(rest >= BN ? BN : round_up((size_t)rest, 32));
    p.idesc = i8_idesc(BM * CTAS, BN);
    p.idesc_last = i8_idesc(BM * CTAS, p.n_last);
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
    QNN_REQUIRE(tiles < ((int64_t)1 << 31), QNN_ERR_UNSUPPORTED, "qnn_gemm_i8_scaled: too many output tiles");
    const int64_t nw = tiles < workers ? tiles : workers;
    profile_before(st);
    QNN_CUDA(launch_clustered(kern, (unsigned)(CTAS * nw), S::THREADS, S::TOTAL, CTAS, st, ma, mb, mo, p));
    profile_after(st);
    return check_launch("qnn_gemm_i8_scaled");
}

// CTA pairs a persistent grid can keep resident at once, asked once per device (0 = pairs cannot be launched)
int pairs_resident()
{
    static std::atomic<int> cached[64];                 // 0 = not asked yet; stored as pairs + 1
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int v = cached[dev].load(std::memory_order_acquire);
    if (v == 0) {
        using S = WideCfg<256, 2, __nv_bfloat16, 2>;
        auto kern = gemm_i8s_wide_kernel<256, 2, __nv_bfloat16, 2>;
        int n = 0;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::TOTAL) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(2 * (unsigned)sm_count());
            cfg.blockDim = dim3(S::THREADS);
            cfg.dynamicSmemBytes = S::TOTAL;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr; cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) { (void)cudaGetLastError(); n = 0; }
        }
        v = n + 1;
        cached[dev].store(v, std::memory_order_release);
    }
    return v - 1;
}

// Clusters of `split` CTAs of the narrow kernel for up to 128 tokens, one CTA an SM, that are resident at once: SMs / split less
// what the GPU's groups of SMs leave over (eights: 15 of 18, fours: 33 of 37).  Asked for once per device.
template <int SPLIT>
int narrow_clusters_of()
{
    static std::atomic<int> cached[64];                 // 0 = not asked yet
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int v = cached[dev].load(std::memory_order_acquire);
    if (v == 0) {
        using S = NarrowCfg<128>;
        auto kern = gemm_i8s_narrow_kernel<128, __nv_bfloat16, SPLIT>;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::TOTAL) == cudaSuccess) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(SPLIT * (unsigned)sm_count());
            cfg.blockDim = dim3(NARROW_THREADS);
            cfg.dynamicSmemBytes = S::TOTAL;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = SPLIT; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr; cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&v, kern, &cfg) != cudaSuccess) { (void)cudaGetLastError(); v = 0; }
        }
        if (v < 1) v = 1;
        cached[dev].store(v, std::memory_order_release);
    }
    return v;
}
int narrow_clusters(int split)
{
    switch (split) {
        case 1: return sm_count();
        case 2: return narrow_clusters_of<2>();
        case 4: return narrow_clusters_of<4>();
        default: return narrow_clusters_of<8>();
    }
}

template <int MT, int GEMV_R, int GEMV_U, typename TOUT>
int launch_gemv(const I8sCall &c, const I8sParams &p, cudaStream_t st)
{
    // K is cut until there are about sixteen warps for every SM (or a warp's part is a single round of loads)
    const int64_t groups = ceil_div(p.N, GEMV_R);
    int ksplit = 1;
    while (ksplit < 8 && groups * ksplit * 2 <= 16 * (int64_t)sm_count() && c.K / (ksplit * 2) >= 512) ksplit *= 2;
    const int64_t blocks = ceil_div(groups, 8 / ksplit);
    QNN_REQUIRE(blocks < ((int64_t)1 << 31), QNN_ERR_UNSUPPORTED, "qnn_gemm_i8_scaled: too many output channels");
    profile_before(st);
    QNN_CUDA(launch_pdl(gemv_i8s_kernel<MT, GEMV_R, GEMV_U, TOUT>, dim3((unsigned)blocks), dim3(256), 0, st, static_cast<const uint8_t *>(c.a), c.lda,
                        static_cast<const uint8_t *>(c.b), c.ldb, (int32_t)c.K, ksplit, p));
    profile_after(st);
    return check_launch("qnn_gemm_i8_scaled");
}

// The kernel that a product runs on.
struct I8sChoice {
    int kind;                        // QNN_I8S_*; 0: no kernel of these (K = 0)
    int cols;                        // tokens of a thread / columns of a tile
    int split;                       // rows of weights a warp / CTAs that share K / CTAs that share a tile
};
I8sChoice choose_i8s(int64_t M, int64_t N, int64_t K)
{
    if (K == 0) return {0, 0, 0};
    const int32_t num_kb = (int32_t)ceil_div(K, BKB);
    // A handful of tokens: the weights go through the integer units.  One token always (4096 x 4096: 2.8 us against 4.9 us on the
    // tensor cores, 28672 x 4096: 20.9 against 21.4; rows of at most 1024 codes four to a warp: 131072 x 1024 22.7 against
    // 30.5 us two to a warp).  Two to four tokens while the weights are at most 32 MB (two: 4096 x 4096 3.2 against 4.9, but
    // 131072 x 1024 34.4 against 29.2; four: 4096 x 4096 3.5 against 4.9, 11008 x 2048 4.9 against 5.7, but 16384 x 4096 20.3
    // against 14.8), three and four not for the shortest rows (16384 x 512: 4.8 against 4.0).  Eight tokens: 5.9 us for 4096 x
    // 4096.  (Weights of up to 32 MB in L2; 4096 x 4096 from HBM: one token 5.2 us, two 5.9, four 6.1, eight on the tensor cores 5.9.)
    if (M == 1) return {QNN_I8S_TOKENS, 1, K <= 1024 ? 4 : 2};
    if (M <= 4 && N * K <= (int64_t)32 << 20) {
        if (M == 2) return {QNN_I8S_TOKENS, 2, 4};
        if (K >= 1024) return {QNN_I8S_TOKENS, 4, 4};
    }

    // On the tensor cores the time of a launch is roughly, over M = 3 .. 4096, N = 128 .. 131072, K = 128 .. 16384,
    //   wide    start + waves * (K blocks * block + hand-over)
    //   narrow  waves * start + (K blocks of a CTA) * max(block, CTAs an SM * stream) + hand-over      (us, fitted to sweeps)
    // with the constants below; the cheapest configuration runs.  Of 300 random sizes, measured over predicted: narrow 0.8 to 1.3
    // (median 0.99, 5 to 95 %), wide 1.0 to 2.1 (median 1.14, the largest 3.1: a K block or two and large results, whose stores the
    // model does not have -- 273 x 102905 x 211 takes 36 to 50 us and is taken for 16).  It ranks the configurations, and does no more.
    // (Figures here and below: weights of up to 32 MB in L2.)  100 x 4096 x 4096: narrow 7.6, wide 64 columns 9.2;
    // 100 x 11008 x 2048: narrow 9.8, wide 128 columns 7.7; 16 x 131072 x 4096: narrow 85, wide 116 .. 200; 701 x 2047 x 1111:
    // wide 64 columns 8.2, 128 columns 6.6, pairs of 256 columns 9.2; 701 x 4096 x 4096: 22.8, 19.8, and pairs of 128 / 192 / 256
    // columns 18.1 / 13.2 / 15.1.
    struct Config { int rows, cols; float start, block, hand; };            // us
    static const Config wide[] = {{128, 64, 3.2f, 0.21f, 0.1f}, {128, 128, 3.7f, 0.27f, 0.2f}, {256, 128, 4.2f, 0.235f, 0.3f},
                                  {256, 192, 4.8f, 0.285f, 0.5f}, {256, 256, 5.5f, 0.34f, 0.7f}};
    const int sms = sm_count(), pairs = pairs_resident();
    int best = -1;
    float cost = 0.0f;
    for (int i = 0; i < 5; ++i) {
        const int workers = wide[i].rows == 128 ? sms : pairs;
        if (workers < 1) continue;
        const int64_t tiles = ceil_div(M, wide[i].rows) * ceil_div(N, wide[i].cols);
        const float t = wide[i].start + (float)ceil_div(tiles, workers) * (wide[i].block * (float)num_kb + wide[i].hand);
        if (best < 0 || t < cost) { best = i; cost = t; }
    }
    {
        // narrow tiles, K cut until the CTAs are about one for every SM: few tokens, or few channels and a long K.  The weights
        // (and with many CTAs an SM nothing else) set the pace; wide tiles stream them less well, which counts when all that
        // there is to do is to stream them.  128 columns have one CTA an SM: K is cut while all clusters are resident at once
        // (100 x 2048 x 4096: 7.2 us in 16 clusters of four, 11.9 in 16 of eight, of which 15 fit).
        struct Narrow { int cols; float start, block, stream, hand; };
        static const Narrow narrow[] = {{16, 3.0f, 0.28f, 0.34f, 0.3f}, {32, 3.5f, 0.31f, 0.28f, 0.3f}, {64, 4.0f, 0.22f, 0.38f, 0.3f},
                                        {128, 5.0f, 0.31f, 0.46f, 0.6f}};
        const int i = M <= 16 ? 0 : M <= 32 ? 1 : M <= 64 ? 2 : 3;
        const int64_t tiles = ceil_div(N, BM) * ceil_div(M, narrow[i].cols);
        int split = 1;
        while (split < 8 && num_kb / (split * 2) >= 2 &&
               (i == 3 ? tiles <= narrow_clusters(split * 2) : tiles * split * 2 <= (int64_t)sms * 5 / 4)) split *= 2;
        const int64_t waves = i == 3 ? ceil_div(tiles, narrow_clusters(split)) : ceil_div(tiles * split, 2 * sms);
        const int64_t ctas = tiles * split;
        const float an_sm = (float)ctas / (float)sms * narrow[i].stream;
        const float t = (float)waves * narrow[i].start +
                        (float)ceil_div(num_kb, split) * (an_sm > narrow[i].block ? an_sm : narrow[i].block) + (split > 1 ? narrow[i].hand : 0.0f);
        if (M <= 128) {
            const float stream = 4.0f + 1.35f * (float)(N * K) * 1e-6f / 6.5f;   // (6.5 MB a us)
            if (cost < stream) cost = stream;
        }
        if (t < cost) return {QNN_I8S_NARROW, narrow[i].cols, split};
    }
    return {QNN_I8S_WIDE, wide[best].cols, wide[best].rows / BM};
}

template <typename TOUT>
int run_i8s(const I8sCall &c, const I8sParams &p, cudaStream_t st)
{
    const I8sChoice k = choose_i8s(p.M, p.N, c.K);
    switch (k.kind) {
        case QNN_I8S_TOKENS:
            if (k.cols == 1) return k.split == 4 ? launch_gemv<1, 4, 1, TOUT>(c, p, st) : launch_gemv<1, 2, 4, TOUT>(c, p, st);
            return k.cols == 2 ? launch_gemv<2, 4, 1, TOUT>(c, p, st) : launch_gemv<4, 4, 4, TOUT>(c, p, st);
        case QNN_I8S_NARROW:
            switch (k.cols) {
                case 16: return launch_narrow<16, TOUT>(c, p, k.split, st);
                case 32: return launch_narrow<32, TOUT>(c, p, k.split, st);
                case 64: return launch_narrow<64, TOUT>(c, p, k.split, st);
                default: return launch_narrow<128, TOUT>(c, p, k.split, st);
            }
        case QNN_I8S_WIDE:
            if (k.split == 1) return k.cols == 64 ? launch_wide<64, 1, TOUT>(c, p, sm_count(), st) : launch_wide<128, 1, TOUT>(c, p, sm_count(), st);
            switch (k.cols) {
                case 128: return launch_wide<128, 2, TOUT>(c, p, pairs_resident(), st);
                case 192: return launch_wide<192, 2, TOUT>(c, p, pairs_resident(), st);
                default: return launch_wide<256, 2, TOUT>(c, p, pairs_resident(), st);
            }
        default: {
            const int64_t need = ceil_div(p.M * p.N, 256), cap = (int64_t)sm_count() * 32;
            QNN_CUDA(launch_pdl(bias_rows_kernel<TOUT>, dim3((unsigned)(need < cap ? need : cap)), dim3(256), 0, st, p.M, p.N, p.bias,
                                static_cast<TOUT *>(p.out), p.ldo));
            return check_launch("qnn_gemm_i8_scaled");
        }
    }
}

}  // namespace

int gemm_i8s_selftest(uint8_t *scratch, cudaStream_t st)
{
    // 16 tokens of 512 codes and 128 channels: four CTAs, a K block each
    I8sParams p{};
    p.M = 16; p.N = BM; p.num_kb = 4; p.tiles_n = p.tiles_m = 1;
    const I8sCall c = {scratch, scratch + 16 * 512, 512, 512, 512};
    float *f = reinterpret_cast<float *>(scratch + (16 + BM) * 512);
    p.a_scale = f; p.b_scale = f + 16;
    p.out = f + 16 + BM; p.ldo = BM;
    static_assert((16 + BM) * 512 + (16 + BM + 16 * BM) * 4 <= CLUSTER_SELFTEST_BYTES, "scratch");
    return launch_narrow_split<16, float, 4, true>(c, p, st);
}

int gemm_i8s_status(int *code)
{
    QNN_CUDA(status_read_clear(code));
    return QNN_OK;
}

}  // namespace qnn

using namespace qnn;

extern "C" int qnn_gemm_i8_scaled_kernel(int64_t M, int64_t N, int64_t K)
{
    if (M <= 0 || N <= 0 || K < 0 || M > (int64_t)1 << 30 || N > (int64_t)1 << 30 || K >= (int64_t)1 << 17) return 0;
    const I8sChoice k = choose_i8s(M, N, K);
    return k.kind | k.cols << 4 | k.split << 16;
}

extern "C" int qnn_gemm_i8_scaled(const void *a, int64_t lda, const float *a_scale, const void *b, int64_t ldb, const float *b_scale,
                                  const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_type, int64_t ldo, void *stream)
{
    const char *what = "qnn_gemm_i8_scaled";
    QNN_REQUIRE(type_ok(out_type), QNN_ERR_INVALID_ARG, "%s: unknown output type %d", what, out_type);
    QNN_REQUIRE(M >= 0 && N >= 0 && K >= 0, QNN_ERR_INVALID_ARG, "%s: negative size", what);
    QNN_REQUIRE(M <= (int64_t)1 << 30 && N <= (int64_t)1 << 30, QNN_ERR_UNSUPPORTED, "%s: M or N above 2^30", what);
    QNN_REQUIRE(K < (int64_t)1 << 17, QNN_ERR_OVERFLOW, "%s: K of 2^17 and more: 128 * 128 * K does not fit int32", what);
    if (M == 0 || N == 0) return QNN_OK;
    QNN_REQUIRE(a_scale && b_scale && out && (K == 0 || (a && b)), QNN_ERR_INVALID_ARG, "%s: NULL pointer", what);
    QNN_REQUIRE(ldo >= N, QNN_ERR_INVALID_ARG, "%s: ldo below N", what);
    QNN_REQUIRE(aligned(out, (size_t)type_bytes(out_type)) && aligned(a_scale, 4) && aligned(b_scale, 4) && aligned(bias, 4), QNN_ERR_ALIGNMENT,
                "%s: a pointer is not aligned to its elements", what);
    if (K > 0) {
        QNN_REQUIRE(lda >= K && ldb >= K, QNN_ERR_INVALID_ARG, "%s: lda or ldb below K", what);
        QNN_REQUIRE(aligned(a, 16) && aligned(b, 16) && lda % 16 == 0 && ldb % 16 == 0, QNN_ERR_ALIGNMENT,
                    "%s: codes must be 16-byte aligned, lda and ldb multiples of 16", what);
    }
    I8sParams p{};
    p.M = M; p.N = N; p.num_kb = (int32_t)ceil_div(K, BKB);
    p.a_scale = a_scale; p.b_scale = b_scale; p.bias = bias;
    p.out = out; p.ldo = ldo;
    const I8sCall c = {a, b, lda, ldb, K};
    cudaStream_t st = as_stream(stream);
    switch (out_type) {
        case QNN_TYPE_F32: return run_i8s<float>(c, p, st);
        case QNN_TYPE_BF16: return run_i8s<__nv_bfloat16>(c, p, st);
        default: return run_i8s<__half>(c, p, st);
    }
}
