// int8 x int8 product with a scale for each token and each output channel:
//   out[m, n] = (float(sum_k a[m,k] b[n,k]) * a_scale[m]) * b_scale[n] + bias[n]
// The sum is exact in int32 (tcgen05 kind::i8 accumulates there), so it does not depend on tiles or splits.
//
// Two kernels:
//  - wide: persistent; tokens are the tile's 128 (a CTA pair: 256) rows, channels its columns.  Warp 0 loads by TMA, warp 1
//    multiplies into one of two accumulator stages in tensor memory, the other warps scale and store the previous tile.
//  - narrow, for few tokens: bound by the bytes of the weights, so weights are the tile's 128 rows and the tokens its 16..128
//    columns; K is cut among the CTAs of a cluster, whose int32 partial sums meet in shared memory.
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
        int32_t tn_parked = -1;
        for (uint32_t t = blockIdx.x / CTAS; t < num_tiles && ok; t += gridDim.x / CTAS, ++iter) {
            const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
            const int64_t ntile = (int64_t)tn * BN;
            const int64_t m0 = ((int64_t)tm * CTAS + rank) * BM + q * 32;       // the row of the warp's lane 0
            const float sa = m0 + lane < p.M ? __ldg(p.a_scale + m0 + lane) : 0.0f;
            if (tn != tn_parked) {                               // consecutive tiles mostly share their columns
                tn_parked = tn;
                __syncwarp();
                for (int b = 0; b < S::NBW; ++b) {
                    for (int c = lane; c < S::CB; c += 32) {
                        const int blk = grp + b * G;
                        const int64_t n = ntile + blk * S::CB + c;
                        const bool in = blk < S::NB && n < p.N;
                        cs[b * S::CB + c] = in ? __ldg(p.b_scale + n) : 0.0f;
                        cb[b * S::CB + c] = (in && p.bias) ? __ldg(p.bias + n) : 0.0f;
                    }
                }
                __syncwarp();
            }
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
                    TOUT *dst = static_cast<TOUT *>(p.out) + m0 * p.ldo + n0;
#pragma unroll 4
                    for (int r = 0; r < rows; ++r) {
#pragma unroll
                        for (int h = 0; h < S::CB / 32; ++h) {
                            const int c = h * 32 + lane;
                            const int byte = c * (int)sizeof(TOUT);
                            const TOUT x = *reinterpret_cast<const TOUT *>(stg + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15));
                            if (n0 + c < p.N) dst[(int64_t)r * p.ldo + c] = x;
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
            tm += (int32_t)step_m; tn += (int32_t)step_n;
            if (tm >= (int32_t)tiles_m) { tm -= (int32_t)tiles_m; ++tn; }
        }
        if (lane == 0) bulk_wait_all();                          // stores must have read shared memory before it goes away
        __syncwarp();
    }

    __syncwarp();
    if (*abort_flag) {
        // give copies and products still in flight time to land before shared and tensor memory are released
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
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
    // two CTAs fit an SM: one CTA's set-up and join overlap the other's stream of weights
    static constexpr int STAGES = (108 * 1024) / STAGE_BYTES > 6 ? 6 : (108 * 1024) / STAGE_BYTES;
    static constexpr int BAR_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int TOTAL = BAR_OFFSET + 128 + 1024;
    static constexpr int TMEM = tmem_cols(BN);
    static_assert(STAGES * STAGE_BYTES >= BN * BM * 4, "the partial sums reuse the stages");
    static_assert((2 * STAGES + 1) * 8 + 8 <= 128, "barriers");
};

__device__ __forceinline__ int32_t ld_peer_i32(uint32_t addr)
{
    int32_t v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

template <int BN, typename TOUT>
__global__ void __launch_bounds__(NARROW_THREADS, 2)
gemm_i8s_narrow_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const I8sParams p,
                       const int split)
{
    using S = NarrowCfg<BN>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *gen = smem_raw + (base - raw);
    const uint32_t bar0 = base + S::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(S::STAGES + s); };
    const uint32_t done_bar = bar0 + 8u * (uint32_t)(2 * S::STAGES);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gen + S::BAR_OFFSET + 8 * (2 * S::STAGES + 1));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x % (uint32_t)split;                // = the CTA's rank in its cluster
    const uint32_t tile = blockIdx.x / (uint32_t)split;
    const int32_t tn = (int32_t)(tile % (uint32_t)p.tiles_n), tm = (int32_t)(tile / (uint32_t)p.tiles_n);
    const int32_t kb0 = (int32_t)((int64_t)p.num_kb * rank / split), kb1 = (int32_t)((int64_t)p.num_kb * (rank + 1) / split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        mbar_init(done_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_u32(tmem_slot), S::TMEM);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    griddep_launch_dependents();                                       // (after the allocation, as above)
    griddep_wait();

    const int32_t nt = p.M - (int64_t)tm * BN < BN ? (int32_t)(p.M - (int64_t)tm * BN) : BN;   // tokens of this tile
    int32_t *part = reinterpret_cast<int32_t *>(gen);                  // [token][128 channels], over the operand stages
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
        ok = __all_sync(0xffffffffu, mbar_wait(done_bar, 0, abort_flag, 17));
        if (ok) {
            tc_fence_after();
            const int n_local = q * 32 + lane;
            const int64_t n = (int64_t)tn * BM + n_local;
            const float sb = (split == 1 && n < p.N) ? __ldg(p.b_scale + n) : 0.0f;
            const float bi = (split == 1 && n < p.N && p.bias) ? __ldg(p.bias + n) : 0.0f;
#pragma unroll 1
            for (int c = 0; c < nt; c += 16) {
                uint32_t v[16];
                asm volatile(
                    "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                    "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                    : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                      "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                    : "r"(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)c) : "memory");
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (c + j < nt) {
                        if (split > 1) {
                            part[(c + j) * BM + n_local] = (int32_t)v[j];
                        } else if (n < p.N) {
                            const int64_t m = (int64_t)tm * BN + c + j;
                            const float f = fmaf(__int2float_rn((int32_t)v[j]) * __ldg(p.a_scale + m), sb, bi);
                            from_float(f, static_cast<TOUT *>(p.out)[m * p.ldo + n]);
                        }
                    }
                }
            }
        }
    }
    __syncwarp();
    if (split > 1) {
        // every CTA of the cluster reaches both barriers, whatever became of its waits
        cluster_sync_all();
        if (warp >= 2 && ok) {
            const int n_local = threadIdx.x - 64;
            const int64_t n = (int64_t)tn * BM + n_local;
            if (n < p.N) {
                const float sb = __ldg(p.b_scale + n), bi = p.bias ? __ldg(p.bias + n) : 0.0f;
                for (int j = (int)rank; j < nt; j += split) {
                    const uint32_t at = smem_u32(part + j * BM + n_local);
                    int32_t s = 0;
                    for (int r = 0; r < split; ++r) s += ld_peer_i32(map_to_cta(at, (uint32_t)r));
                    const int64_t m = (int64_t)tm * BN + j;
                    const float f = fmaf(__int2float_rn(s) * __ldg(p.a_scale + m), sb, bi);
                    from_float(f, static_cast<TOUT *>(p.out)[m * p.ldo + n]);
                }
            }
        }
        cluster_sync_all();                // nobody leaves while its partial sums are being read
    }
    if (*abort_flag) {
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc<1>(tmem_base, S::TMEM);
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

int make_map(CUtensorMap *map, CUtensorMapDataType type, int64_t es, const void *base, int64_t rows, int64_t cols, int64_t ld_bytes, int box_rows,
             int box_cols, CUtensorMapL2promotion promo)
{
    EncodeTiledFn fn = encode_fn();
    QNN_REQUIRE(fn != nullptr, QNN_ERR_CUDA, "qnn_gemm_i8_scaled: cuTensorMapEncodeTiled is not available from this driver");
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld_bytes};
    cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    (void)es;
    CUresult r = fn(map, type, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    promo, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    QNN_REQUIRE(r == CUDA_SUCCESS, QNN_ERR_CUDA, "qnn_gemm_i8_scaled: cuTensorMapEncodeTiled failed with code %d", (int)r);
    return QNN_OK;
}
int make_map_codes(CUtensorMap *map, const void *base, int64_t rows, int64_t K, int64_t ld, int box_rows)
{
    return make_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, rows, K, ld, box_rows, BKB, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
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

template <int BN, typename TOUT>
int launch_narrow(const I8sCall &c, I8sParams p, cudaStream_t st)
{
    using S = NarrowCfg<BN>;
    auto kern = gemm_i8s_narrow_kernel<BN, TOUT>;
    static std::atomic<bool> done[64];
    if (int rc = opt_in(kern, S::TOTAL, done)) return rc;
    CUtensorMap mw, mx;
    if (int rc = make_map_codes(&mw, c.b, p.N, c.K, c.ldb, BM)) return rc;
    if (int rc = make_map_codes(&mx, c.a, p.M, c.K, c.lda, BN)) return rc;
    p.tiles_n = (int32_t)ceil_div(p.N, BM);
    p.tiles_m = (int32_t)ceil_div(p.M, BN);
    p.idesc = i8_idesc(BM, BN);
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_m;
    int split = 1;
    while (split < 8 && tiles * split * 2 <= 2 * (int64_t)sm_count() && p.num_kb / (split * 2) >= 2) split *= 2;
    QNN_REQUIRE(tiles * split < ((int64_t)1 << 31), QNN_ERR_UNSUPPORTED, "qnn_gemm_i8_scaled: too many output tiles");
    profile_before(st);
    QNN_CUDA(launch_clustered(kern, (unsigned)(tiles * split), NARROW_THREADS, S::TOTAL, split, st, mw, mx, p, split));
    profile_after(st);
    return check_launch("qnn_gemm_i8_scaled");
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
        if (int rc = make_map(&mo, dt, sizeof(TOUT), p.out, p.M, p.N, p.ldo * (int64_t)sizeof(TOUT), 32, S::CB, CU_TENSOR_MAP_L2_PROMOTION_NONE))
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

template <typename TOUT>
int run_i8s(const I8sCall &c, const I8sParams &p, cudaStream_t st)
{
    if (c.K == 0) {
        const int64_t need = ceil_div(p.M * p.N, 256), cap = (int64_t)sm_count() * 32;
        QNN_CUDA(launch_pdl(bias_rows_kernel<TOUT>, dim3((unsigned)(need < cap ? need : cap)), dim3(256), 0, st, p.M, p.N, p.bias,
                            static_cast<TOUT *>(p.out), p.ldo));
        return check_launch("qnn_gemm_i8_scaled");
    }
    if (p.M <= 16) return launch_narrow<16, TOUT>(c, p, st);
    if (p.M <= 32) return launch_narrow<32, TOUT>(c, p, st);
    if (p.M <= 64) return launch_narrow<64, TOUT>(c, p, st);
    if (p.M <= 128) return launch_narrow<128, TOUT>(c, p, st);
    const int pairs = pairs_resident();
    if (pairs >= 8 && ceil_div(p.M, 256) * ceil_div(p.N, 256) >= pairs) return launch_wide<256, 2, TOUT>(c, p, pairs, st);
    return launch_wide<128, 1, TOUT>(c, p, sm_count(), st);
}

}  // namespace

int gemm_i8s_status(int *code)
{
    QNN_CUDA(status_read_clear(code));
    return QNN_OK;
}

}  // namespace qnn

using namespace qnn;

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
