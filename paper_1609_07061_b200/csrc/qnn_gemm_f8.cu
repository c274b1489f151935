// Products of 8-bit floating-point codes (e4m3, e5m2) with a power-of-two scale for each block of 128 along the reduction:
//   out[m, n]   = sum_k a[m,k] sa[m, k/128] b[g][n,k] sb[g][n/128, k/128] + bias[g][n]        rows m of group g (forward)
//   out[m, n]   = sum_k a[m,k] sa[m, k/128] b[g][k,n] sb[g][k/128, n/128]                      the same weights read across (input gradient)
//   dw[g][n, k] = sum_m y[m,n] sy[m/128, n] x[m,k] sx[m/128, k]                                rows m of group g (weight gradient)
// The dense product is the grouped one with a single group.
//
// The tensor cores apply the scales themselves (tcgen05 kind::mxf8f6f4 with block scales: one byte for 32 elements, here the same
// byte for the four steps of a block), so partial sums never leave tensor memory before a tile is done.
//
// One persistent kernel.  The weights (in a weight gradient: the output's rows) are the tile's 128 rows, the tokens its
// columns: their number is given to the instruction at run time, so a group of 37 rows costs 48 columns and not a tile.  Weights read
// across, and both operands of a weight gradient, are taken as they lie in memory: the tensor core reads them MN-major.
// Warp 0 loads by TMA, warp 1 multiplies into one of two accumulators, warp 2 fetches scales and lays them out for the copy into
// tensor memory, warps 4..7 store the previous tile.  All waits are bounded.
#include <cuda.h>
#include <atomic>
#include "qnn_types.cuh"
#include "qnn_tc_ptx.cuh"

namespace qnn {
namespace {

constexpr int MAX_GROUPS = QNN_F8_MAX_GROUPS;
constexpr int F8_THREADS = 256;
enum Mode { FORWARD = 0, ACROSS = 1, WGRAD = 2 };

struct F8Params {
    int64_t M;                       // rows of a (tokens) of all groups; offsets are held to 0..M
    int32_t N;                       // channels: rows of the tile's operand (forward: n, across: n, weight gradient: n)
    int32_t C;                       // weight gradient: columns (k)
    int32_t nkb;                     // blocks of the reduction (forward, across)
    int32_t groups;
    const int64_t *offsets;          // [groups + 1] or NULL: one group of all rows
    const uint8_t *w_scale; int64_t ld_ws, stride_ws;      // scales of the tile's rows
    const uint8_t *x_scale; int64_t ld_xs;                 // scales of the tile's columns
    const float *bias;               // [groups, N] or NULL
    void *out; int64_t ldo;
    int32_t vec_out;                 // rows of the output may be written in 16-byte pieces
    int32_t tiles_c;                 // tiles of channels
    int32_t chunks, chunk;           // weight gradient: tiles of columns, and columns of each
    int32_t super;                   // chunks of tokens that go through all channels before the next ones
    uint32_t idesc;                  // without N and the scales' byte
};

template <int NT, int MODE, int CTAS, typename TOUT>
struct F8Cfg {
    static constexpr int A_BYTES = BM * BKB;
    static constexpr int BROWS = NT / CTAS > 128 ? 256 : NT / CTAS > 64 ? 128 : NT / CTAS > 32 ? 64 : 32;   // rows (columns, MN-major) a CTA loads at most
    static constexpr int B_BYTES = BROWS * BKB;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int STG_BYTES = 4 * 32 * 32 * (int)sizeof(TOUT);   // a block of 32 x 32 results for each storing warp
    static constexpr int SFB = (NT + 127) / 128;                        // 512-byte pieces of column scales
    static constexpr int SF_BYTES = 512 * (1 + SFB);
    static constexpr int SLOTS = NT > 128 ? 2 : 4;                      // words of scales in flight (four blocks each)
    static constexpr int SF_COLS = 4 + 4 * SFB;                         // tensor-memory columns of one word's scales
    static constexpr int TMEM_NEED = 2 * NT + SLOTS * SF_COLS;
    static constexpr int TMEM = TMEM_NEED <= 128 ? 128 : TMEM_NEED <= 256 ? 256 : 512;
    static constexpr int TABLE_BYTES = 2 * 4 * (MAX_GROUPS + 8);
    static constexpr int AUX = STG_BYTES + SLOTS * SF_BYTES + TABLE_BYTES + 256 + 1024;
    static constexpr int MAXS = (SMEM_LIMIT - AUX) / STAGE_BYTES;
    static constexpr int STAGES = MAXS > 8 ? 8 : MAXS;
    static constexpr int STG_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int SF_OFFSET = STG_OFFSET + STG_BYTES;
    static constexpr int TABLE_OFFSET = SF_OFFSET + SLOTS * SF_BYTES;
    static constexpr int BAR_OFFSET = TABLE_OFFSET + TABLE_BYTES;
    static constexpr int TOTAL = BAR_OFFSET + 256 + 1024;
    static_assert(STAGES >= 3 && TMEM_NEED <= 512 && (2 * STAGES + 2 * SLOTS + 4) * 8 + 16 <= 256 && TOTAL <= SMEM_LIMIT, "configuration");
};

// ---- PTX ---------------------------------------------------------------------------------------------------------

// descriptor of a tile of 128-byte rows, swizzled over 128 bytes, whose ROWS run along the reduction: 8-row groups 1024 bytes apart,
// the next 128 elements of the other dimension 128 rows further on
__device__ __forceinline__ uint64_t make_across_desc(uint32_t saddr)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3ffffu) >> 4);
    d |= (uint64_t)((128 * BKB) >> 4) << 16;
    d |= (uint64_t)((8 * BKB) >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// 32 rows of 16 bytes, one after the other, no swizzle: a piece of scales
__device__ __forceinline__ uint64_t make_scale_desc(uint32_t saddr)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3ffffu) >> 4);
    d |= (uint64_t)(128 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    return d;
}
// one step of 32 elements along the reduction
template <int CTAS>
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    if (CTAS == 2)
        asm volatile("{\n.reg .pred P;\nsetp.ne.b32 P, %6, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], P;\n}\n"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n.reg .pred P;\nsetp.ne.b32 P, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], P;\n}\n"
                     ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// 512 bytes of scales into four tensor-memory columns, the same in each quarter of the lanes
template <int CTAS>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc)
{
    if (CTAS == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if (CTAS == 2) umma_commit_pair(bar);
    else umma_commit(bar);
}
template <int CTAS>
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar)
{
    if (CTAS == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar)
{
    if (CTAS == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t a) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(a) : "memory"); }

// ---- tiles -------------------------------------------------------------------------------------------------------

struct F8Tile {
    int32_t g;                       // group
    int32_t c0;                      // first channel (of the pair)
    int32_t m0;                      // first token; weight gradient: first column
    int32_t cols;                    // columns with a result
    int32_t n;                       // columns multiplied: rounded up to what the instruction takes
    int32_t kb;                      // blocks of the reduction
    int32_t blk0;                    // weight gradient: the group's first block of rows
};

// Walks the tiles of one CTA (pair) in rising order; every role of the CTA walks by itself.
template <int NT, int MODE, int CTAS>
struct Tiles {
    const F8Params &p;
    const int32_t *first, *start;    // [groups + 1] first tile / (forward, across) first row or (weight gradient) first block
    int32_t g = 0;
    __device__ __forceinline__ Tiles(const F8Params &p_, const int32_t *f, const int32_t *s) : p(p_), first(f), start(s) {}
    __device__ __forceinline__ int32_t count() const { return first[p.groups]; }
    __device__ __forceinline__ F8Tile at(int32_t t)
    {
        while (t >= first[g + 1]) ++g;
        F8Tile r;
        r.g = g;
        const int32_t i = t - first[g];
        constexpr int STEP = MODE == WGRAD ? 16 * CTAS : 16;
        if (MODE == WGRAD) {
            const int32_t c = i / p.chunks, ch = i - c * p.chunks;
            r.c0 = c * BM * CTAS;
            r.m0 = ch * p.chunk;
            r.cols = p.C - r.m0 < p.chunk ? p.C - r.m0 : p.chunk;
            r.blk0 = start[g];
            r.kb = start[g + 1] - start[g];
        } else {
            const int32_t len = start[g + 1] - start[g];
            const int32_t chunks = (len + NT - 1) / NT;
            const int32_t csize = ((len + chunks - 1) / chunks + STEP - 1) / STEP * STEP;
            const int32_t sup = i / (p.super * p.tiles_c);
            const int32_t j = i - sup * p.super * p.tiles_c;
            const int32_t wide = chunks - sup * p.super < p.super ? chunks - sup * p.super : p.super;
            const int32_t c = j / wide;
            const int32_t ch = sup * p.super + (j - c * wide);
            r.c0 = c * BM * CTAS;
            r.m0 = start[g] + ch * csize;
            r.cols = start[g + 1] - r.m0 < csize ? start[g + 1] - r.m0 : csize;
            r.kb = p.nkb;
            r.blk0 = 0;
        }
        r.n = (r.cols + STEP - 1) / STEP * STEP;
        return r;
    }
};

// first[], start[] in shared memory from the offsets in global memory, by all threads of the block.  Offsets that fall, or leave
// 0..M, are held to rise and to stay inside, so that no group reaches rows that are not there.
template <int NT, int MODE>
__device__ void fill_tables(const F8Params &p, int32_t *first, int32_t *start, int32_t *scratch)
{
    constexpr int PER = (MAX_GROUPS + F8_THREADS) / F8_THREADS;         // offsets a thread: groups + 1 of them at most MAX_GROUPS + 1
    static_assert(PER * F8_THREADS >= MAX_GROUPS + 1, "table");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t G = p.groups;
    int32_t o[PER];
    int32_t top = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int g = tid * PER + i;
        int64_t v = 0;
        if (g <= G) v = p.offsets ? __ldg(p.offsets + g) : (g == 0 ? 0 : p.M);
        v = v < 0 ? 0 : v > p.M ? p.M : v;
        top = (int32_t)v > top ? (int32_t)v : top;
        o[i] = top;
    }
    // running maximum over the threads before
    int32_t run = top;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t v = __shfl_up_sync(0xffffffffu, run, d);
        if (lane >= d && v > run) run = v;
    }
    if (lane == 31) scratch[warp] = run;
    __syncthreads();
    int32_t before = __shfl_up_sync(0xffffffffu, run, 1);
    if (lane == 0) before = 0;
    for (int w = 0; w < warp; ++w) before = scratch[w] > before ? scratch[w] : before;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int g = tid * PER + i;
        if (g <= G) start[g] = o[i] > before ? o[i] : before;
    }
    __syncthreads();
    // tiles (and blocks) of each group, added up
    int32_t tl[PER], bl[PER], tsum = 0, bsum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int g = tid * PER + i;
        const int32_t len = g < G ? start[g + 1] - start[g] : 0;
        tl[i] = tsum; bl[i] = bsum;
        bsum += (len + 127) / 128;
        if (g < G) tsum += MODE == WGRAD ? p.tiles_c * p.chunks : (len + NT - 1) / NT * p.tiles_c;
    }
    int32_t trun = tsum, brun = bsum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t v = __shfl_up_sync(0xffffffffu, trun, d), u = __shfl_up_sync(0xffffffffu, brun, d);
        if (lane >= d) { trun += v; brun += u; }
    }
    if (lane == 31) { scratch[8 + warp] = trun; scratch[16 + warp] = brun; }
    __syncthreads();
    trun -= tsum; brun -= bsum;
    for (int w = 0; w < warp; ++w) { trun += scratch[8 + w]; brun += scratch[16 + w]; }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int g = tid * PER + i;
        if (g <= G) {
            first[g] = trun + tl[i];
            if (MODE == WGRAD) start[g] = brun + bl[i];
        }
    }
    __syncthreads();
}

// ---- the kernel --------------------------------------------------------------------------------------------------

template <int NT, int MODE, int CTAS, typename TOUT>
__global__ void __launch_bounds__(F8_THREADS, 1)
gemm_f8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_x32,
               const F8Params p)
{
    using S = F8Cfg<NT, MODE, CTAS, TOUT>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                      // swizzled tiles need 1024-byte alignment
    uint8_t *gen = smem_raw + (base - raw);
    const uint32_t bar0 = base + S::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(S::STAGES + s); };
    auto sfull_bar = [&](int s) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + s); };
    auto sempty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + S::SLOTS + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + 2 * S::SLOTS + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * S::STAGES + 2 * S::SLOTS + 2 + a); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gen + S::BAR_OFFSET + 8 * (2 * S::STAGES + 2 * S::SLOTS + 4));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int32_t *first = reinterpret_cast<int32_t *>(gen + S::TABLE_OFFSET);
    int32_t *start = first + MAX_GROUPS + 8;

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    // a pair's CTA 0 leads: it owns the full, scales-full and accumulator-empty barriers and issues the products
    const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int s = 0; s < S::SLOTS; ++s) { mbar_init(sfull_bar(s), CTAS); mbar_init(sempty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 4 * CTAS); }
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
    fill_tables<NT, MODE>(p, first, start, reinterpret_cast<int32_t *>(gen + S::STG_OFFSET));

    Tiles<NT, MODE, CTAS> tiles(p, first, start);
    const int32_t num_tiles = tiles.count();
    const int32_t worker = (int32_t)(blockIdx.x / CTAS), workers = (int32_t)(gridDim.x / CTAS);

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0;
            bool ok = true;
            const uint32_t fb0 = (CTAS == 2) ? map_to_cta(full_bar(0), 0) : full_bar(0);
            for (int32_t t = worker; t < num_tiles && ok; t += workers) {
                const F8Tile r = tiles.at(t);
                const int32_t mine = r.n / CTAS;                       // columns this CTA loads
                const int32_t x0 = r.m0 + (int32_t)rank * mine;
                const int32_t c0 = r.c0 + (int32_t)rank * BM;
                // K-major: boxes of 128 rows, the rest in boxes of 32; MN-major: boxes of 128 columns
                const int32_t n32 = (mine + 31) / 32;
                const int32_t big = MODE == WGRAD ? (mine + 127) / 128 : S::BROWS >= 128 ? n32 / 4 + (n32 % 4 == 3 ? 1 : 0) : 0;
                const int32_t small = MODE == WGRAD ? 0 : n32 - 4 * big < 0 ? 0 : n32 - 4 * big;
                const uint32_t bytes = (uint32_t)(S::A_BYTES + big * 128 * BKB + small * 32 * BKB) * CTAS;
                for (int32_t kb = 0; kb < r.kb; ++kb) {
                    if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, 41)) { ok = false; break; }
                    const uint32_t sa = base + (uint32_t)(stage * S::STAGE_BYTES), sb = sa + S::A_BYTES;
                    const uint32_t fb = fb0 + 8u * (uint32_t)stage;
                    if (leader) expect_tx(full_bar(stage), bytes);
                    if (MODE == FORWARD) tma_load_3d<CTAS>(sa, &tmap_w, kb * BKB, c0, r.g, fb);
                    else if (MODE == ACROSS) tma_load_3d<CTAS>(sa, &tmap_w, c0, kb * BKB, r.g, fb);
                    else tma_load_3d<CTAS>(sa, &tmap_w, c0, (r.blk0 + kb) * BKB, 0, fb);
                    for (int32_t i = 0; i < big; ++i) {
                        if (MODE == WGRAD) tma_load_2d<CTAS>(sb + (uint32_t)(i * 128 * BKB), &tmap_x, x0 + i * 128, (r.blk0 + kb) * BKB, fb);
                        else tma_load_2d<CTAS>(sb + (uint32_t)(i * 128 * BKB), &tmap_x, kb * BKB, x0 + i * 128, fb);
                    }
                    for (int32_t i = 0; i < small; ++i)
                        tma_load_2d<CTAS>(sb + (uint32_t)((big * 128 + i * 32) * BKB), &tmap_x32, kb * BKB, x0 + big * 128 + i * 32, fb);
                    if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            int stage = 0, slot = 0; uint32_t phase = 0, sphase = 0, iter = 0;
            bool ok = true;
            // a step of 32 along the reduction: 32 bytes of a K-major row, 32 rows of an MN-major tile
            constexpr uint32_t A_STEP = MODE == FORWARD ? 2 : (32 * BKB) >> 4, B_STEP = MODE == WGRAD ? (32 * BKB) >> 4 : 2;
            for (int32_t t = worker; t < num_tiles && ok; t += workers, ++iter) {
                const F8Tile r = tiles.at(t);
                const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
                if (!mbar_wait(tempty_bar(as), aphase ^ 1u, abort_flag, 42)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + as * (uint32_t)NT;
                const uint32_t idesc = p.idesc | (uint32_t)(r.n >> 3) << 17;
                uint32_t sfa = 0, sfb = 0;
                for (int32_t kb = 0; kb < r.kb; ++kb) {
                    if ((kb & 3) == 0) {
                        if (!mbar_wait(sfull_bar(slot), sphase, abort_flag, 43)) { ok = false; break; }
                        tc_fence_after();
                        sfa = tmem_base + 2u * NT + (uint32_t)(slot * S::SF_COLS);
                        sfb = sfa + 4u;
                        const uint32_t src = base + (uint32_t)(S::SF_OFFSET + slot * S::SF_BYTES);
                        copy_scales<CTAS>(sfa, make_scale_desc(src));
#pragma unroll
                        for (int i = 0; i < S::SFB; ++i) copy_scales<CTAS>(sfb + 4u * (uint32_t)i, make_scale_desc(src + 512u * (uint32_t)(1 + i)));
                    }
                    if (!mbar_wait(full_bar(stage), phase, abort_flag, 44)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = base + (uint32_t)(stage * S::STAGE_BYTES), sb = sa + S::A_BYTES;
                    const uint64_t ad = MODE == FORWARD ? make_kmajor_desc<BKB>(sa) : make_across_desc(sa);
                    const uint64_t bd = MODE == WGRAD ? make_across_desc(sb) : make_kmajor_desc<BKB>(sb);
                    const uint32_t id = idesc | (uint32_t)(kb & 3) << 29 | (uint32_t)(kb & 3) << 4;
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)
                        umma_f8<CTAS>(d_tmem, ad + k * A_STEP, bd + k * B_STEP, id, sfa, sfb, (uint32_t)(kb != 0 || k != 0));
                    commit<CTAS>(empty_bar(stage));
                    if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
                    if ((kb & 3) == 3 || kb == r.kb - 1) {
                        commit<CTAS>(sempty_bar(slot));
                        if (++slot == S::SLOTS) { slot = 0; sphase ^= 1u; }
                    }
                }
                if (ok) commit<CTAS>(tfull_bar(as));                   // accumulator complete
            }
        }
    } else if (warp == 2) {
        // Scales: a word holds four blocks' bytes.  Row r of a piece of 128 sits at (r % 32) * 16 + (r / 32) * 4.
        int slot = 0; uint32_t phase = 0;
        bool ok = true;
        auto hand_over = [&]() {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) {
                if (CTAS == 2) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_to_cta(sfull_bar(slot), 0)) : "memory");
                else mbar_arrive(sfull_bar(slot));
            }
            if (++slot == S::SLOTS) { slot = 0; phase ^= 1u; }
        };
        for (int32_t t = worker; t < num_tiles && ok; t += workers) {
            const F8Tile r = tiles.at(t);
            const int32_t c0 = r.c0 + (int32_t)rank * BM;
            if constexpr (MODE == WGRAD) {
                constexpr int PIECES = 1 + S::SFB;
                uint32_t v[PIECES][4];
                auto fetch = [&](int32_t kb) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        const uint8_t *src = i == 0 ? p.w_scale : p.x_scale;
                        const int64_t ld = i == 0 ? p.ld_ws : p.ld_xs;
                        const int32_t col = i == 0 ? c0 + 4 * lane : r.m0 + (i - 1) * 128 + 4 * lane, cols = i == 0 ? p.N : p.C;
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            v[i][b] = col < cols && kb + b < r.kb ? __ldg(reinterpret_cast<const uint32_t *>(src + (int64_t)(r.blk0 + kb + b) * ld + col)) : 0u;
                    }
                };
                if (r.kb > 0) fetch(0);
                for (int32_t kb = 0; kb < r.kb; kb += 4) {
                    uint32_t w[PIECES][4];
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        const uint32_t lo0 = __byte_perm(v[i][0], v[i][1], 0x5140), hi0 = __byte_perm(v[i][0], v[i][1], 0x7362);
                        const uint32_t lo1 = __byte_perm(v[i][2], v[i][3], 0x5140), hi1 = __byte_perm(v[i][2], v[i][3], 0x7362);
                        w[i][0] = __byte_perm(lo0, lo1, 0x5410); w[i][1] = __byte_perm(lo0, lo1, 0x7632);
                        w[i][2] = __byte_perm(hi0, hi1, 0x5410); w[i][3] = __byte_perm(hi0, hi1, 0x7632);
                    }
                    if (kb + 4 < r.kb) fetch(kb + 4);
                    if (!__all_sync(0xffffffffu, mbar_wait(sempty_bar(slot), phase ^ 1u, abort_flag, 45))) { ok = false; break; }
                    const uint32_t dst = base + (uint32_t)(S::SF_OFFSET + slot * S::SF_BYTES);
#pragma unroll
                    for (int i = 0; i < PIECES; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int row = 4 * lane + j;
                            sts32(dst + (uint32_t)(i * 512 + (row % 32) * 16 + (row / 32) * 4), w[i][j]);
                        }
                    hand_over();
                }
            } else {
                constexpr int R = (NT + 31) / 32;                      // rows of tokens a lane
                const uint8_t *ws = p.w_scale + (int64_t)r.g * p.stride_ws;
                const int32_t ct = c0 / BM;
                const bool has_ct = c0 < p.N;                          // (a pair's second half may lie beyond the channels)
                uint4 x[R], xn[R], a, an;
                auto fetch = [&](int32_t kb, uint4 (&xs)[R], uint4 &as) {
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        xs[i] = 32 * i + lane < r.cols ? __ldg(reinterpret_cast<const uint4 *>(p.x_scale + (int64_t)(r.m0 + 32 * i + lane) * p.ld_xs + kb))
                                                       : make_uint4(0, 0, 0, 0);
                    if (MODE == FORWARD) {
                        as = has_ct ? __ldg(reinterpret_cast<const uint4 *>(ws + (int64_t)ct * p.ld_ws + kb)) : make_uint4(0, 0, 0, 0);
                    } else {
                        as = make_uint4(0, 0, 0, 0);
                        if (lane < 16 && has_ct && kb + lane < r.kb) as.x = ws[(int64_t)(kb + lane) * p.ld_ws + ct];
                    }
                };
                if (r.kb > 0) fetch(0, x, a);
                for (int32_t kb = 0; kb < r.kb && ok; kb += 16) {
                    if (kb + 16 < r.kb) fetch(kb + 16, xn, an);
                    uint32_t aw[4];
                    if (MODE == FORWARD) { aw[0] = a.x; aw[1] = a.y; aw[2] = a.z; aw[3] = a.w; }
                    else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            aw[j] = 0;
#pragma unroll
                            for (int b = 0; b < 4; ++b) aw[j] |= __shfl_sync(0xffffffffu, a.x, 4 * j + b) << (8 * b);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (kb + 4 * j >= r.kb) break;
                        if (!__all_sync(0xffffffffu, mbar_wait(sempty_bar(slot), phase ^ 1u, abort_flag, 45))) { ok = false; break; }
                        const uint32_t dst = base + (uint32_t)(S::SF_OFFSET + slot * S::SF_BYTES) + (uint32_t)lane * 16u;
                        sts128(dst, aw[j], aw[j], aw[j], aw[j]);
                        uint32_t w[4 * S::SFB];
#pragma unroll
                        for (int i = 0; i < 4 * S::SFB; ++i) w[i] = i < R ? (j == 0 ? x[i < R ? i : 0].x : j == 1 ? x[i < R ? i : 0].y : j == 2 ? x[i < R ? i : 0].z : x[i < R ? i : 0].w) : 0u;
#pragma unroll
                        for (int i = 0; i < S::SFB; ++i) sts128(dst + 512u * (uint32_t)(1 + i), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                        hand_over();
                    }
#pragma unroll
                    for (int i = 0; i < R; ++i) x[i] = xn[i];
                    a = an;
                }
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3;                                        // tensor-memory lane quarter this warp may read
        uint8_t *stg = gen + S::STG_OFFSET + q * 32 * 32 * (int)sizeof(TOUT);
        constexpr int EPV = 16 / (int)sizeof(TOUT);                    // elements of a 16-byte piece
        constexpr int PIECES = 32 / EPV;                               // pieces of a staged row
        constexpr int PITCH = 32 * (int)sizeof(TOUT);
        // 16-byte pieces of a staged row change places with the row, so that rows written by 32 lanes at once meet in no bank
        auto swz = [](int row, int piece) { return sizeof(TOUT) == 4 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3); };
        uint32_t iter = 0;
        for (int32_t t = worker; t < num_tiles; t += workers, ++iter) {
            const F8Tile r = tiles.at(t);
            const uint32_t as = iter & 1u, aphase = (iter >> 1) & 1u;
            const int32_t ch = r.c0 + (int32_t)rank * BM + q * 32;     // the channel of the warp's lane 0
            const float bias = MODE != WGRAD && p.bias && ch + lane < p.N ? __ldg(p.bias + (int64_t)r.g * p.N + ch + lane) : 0.0f;
            // the tensor-memory loads below are warp-collective: leave the loop only as a whole warp
            if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(as), aphase, abort_flag, 46))) break;
            tc_fence_after();
            const uint32_t tacc = tmem_base + ((uint32_t)(q * 32) << 16) + as * (uint32_t)NT;
            const int32_t nblk = ch < p.N ? (r.cols + 31) / 32 : 0;    // (warp-uniform)
            for (int32_t b = 0; b < nblk; ++b) {
                uint32_t v[32];
                float f[32];
                if (r.kb > 0) tmem_ld32(tacc + (uint32_t)(b * 32), v);
#pragma unroll
                for (int j = 0; j < 32; ++j) f[j] = r.kb > 0 ? __uint_as_float(v[j]) + bias : bias;
                __syncwarp();                                          // the block before has been read
                if (MODE == WGRAD) {
                    // lanes are rows of the output
#pragma unroll
                    for (int c = 0; c < PIECES; ++c) {
                        uint4 o;
                        if constexpr (sizeof(TOUT) == 4)
                            o = make_uint4(__float_as_uint(f[4 * c]), __float_as_uint(f[4 * c + 1]), __float_as_uint(f[4 * c + 2]), __float_as_uint(f[4 * c + 3]));
                        else
                            o = make_uint4(pack2(f[8 * c], f[8 * c + 1], TOUT()), pack2(f[8 * c + 2], f[8 * c + 3], TOUT()),
                                           pack2(f[8 * c + 4], f[8 * c + 5], TOUT()), pack2(f[8 * c + 6], f[8 * c + 7], TOUT()));
                        *reinterpret_cast<uint4 *>(stg + lane * PITCH + swz(lane, c) * 16) = o;
                    }
                } else {
                    // lanes are channels, next to each other in the output's rows
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        TOUT o;
                        from_float(f[j], o);
                        *reinterpret_cast<TOUT *>(stg + j * PITCH + swz(j, lane / EPV) * 16 + (lane % EPV) * (int)sizeof(TOUT)) = o;
                    }
                }
                __syncwarp();
                // the staged block: `rows` rows of `cols` elements at dst
                const int32_t rows_left = MODE == WGRAD ? p.N - ch : r.cols - b * 32, cols_left = MODE == WGRAD ? r.cols - b * 32 : p.N - ch;
                const int rows = rows_left < 32 ? rows_left : 32, cols = cols_left < 32 ? cols_left : 32;
                TOUT *dst = static_cast<TOUT *>(p.out) + (MODE == WGRAD ? ((int64_t)r.g * p.N + ch) * p.ldo + r.m0 + b * 32
                                                                        : (int64_t)(r.m0 + b * 32) * p.ldo + ch);
                if (p.vec_out && cols == 32) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        const int row = i * (32 / PIECES) + lane / PIECES, c = lane % PIECES;
                        const uint4 o = *reinterpret_cast<const uint4 *>(stg + row * PITCH + swz(row, c) * 16);
                        if (row < rows) *reinterpret_cast<uint4 *>(dst + (int64_t)row * p.ldo + c * EPV) = o;
                    }
                } else {
                    TOUT *d = dst + lane;
#pragma unroll 4
                    for (int row = 0; row < rows; ++row, d += p.ldo) {
                        const TOUT o = *reinterpret_cast<const TOUT *>(stg + row * PITCH + swz(row, lane / EPV) * 16 + (lane % EPV) * (int)sizeof(TOUT));
                        if (lane < cols) *d = o;
                    }
                }
            }
            // all reads of this accumulator are done: hand it back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CTAS == 2) mbar_arrive_cluster(map_to_cta(tempty_bar(as), 0));
                else mbar_arrive(tempty_bar(as));
            }
        }
    }

    __syncwarp();
    if (*abort_flag) let_flights_land();
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();     // the peer no longer touches this CTA's barriers, shared or tensor memory
    tc_fence_after();
    if (warp == 1) tmem_dealloc<CTAS>(tmem_base, S::TMEM);
}

// ---- host --------------------------------------------------------------------------------------------------------

struct F8Call {
    const char *what;
    const void *w; int w_type; int64_t w_rows, w_cols, ld_w, stride_w;      // as they lie in memory, `groups` of them stride_w bytes apart
    int32_t w_count;
    const void *x; int x_type; int64_t x_rows, x_cols, ld_x;
};

int make_map_f8(const char *what, CUtensorMap *map, const void *ptr, int64_t cols, int64_t rows, int64_t count, int64_t ld, int64_t stride, int box_rows,
                bool three)
{
    EncodeTiledFn fn = encode_fn();
    QNN_REQUIRE(fn != nullptr, QNN_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available from this driver", what);
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count};
    cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)stride};
    cuuint32_t box[3] = {BKB, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, three ? 3 : 2, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    QNN_REQUIRE(r == CUDA_SUCCESS, QNN_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed with code %d", what, (int)r);
    return QNN_OK;
}

// The shared-memory opt-in is per kernel and device and costs microseconds: asked for once each.
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

template <int NT, int MODE, int CTAS, typename TOUT>
int launch_f8(const F8Call &c, F8Params p, cudaStream_t st)
{
    using S = F8Cfg<NT, MODE, CTAS, TOUT>;
    auto kern = gemm_f8_kernel<NT, MODE, CTAS, TOUT>;
    p.tiles_c = (int32_t)ceil_div(p.N, BM * CTAS);
    if (MODE == WGRAD) {
        p.chunks = (int32_t)ceil_div(p.C, NT);
        p.chunk = (int32_t)round_up((size_t)ceil_div(p.C, p.chunks), 16 * CTAS);
    }
    p.super = 16;
    const int64_t tiles = MODE == WGRAD ? (int64_t)p.groups * p.tiles_c * p.chunks : (ceil_div(p.M, NT) + p.groups) * p.tiles_c;
    QNN_REQUIRE(tiles < (int64_t)1 << 31, QNN_ERR_UNSUPPORTED, "%s: too many output tiles", c.what);
    static std::atomic<bool> done[64];
    if (int rc = opt_in(kern, S::TOTAL, done)) return rc;
    CUtensorMap mw, mx, mx32;
    // (an empty reduction loads nothing: any map will do)
    const bool empty = c.w_rows == 0 || c.w_cols == 0 || c.x_rows == 0 || c.x_cols == 0;
    if (!empty) {
        if (int rc = make_map_f8(c.what, &mw, c.w, c.w_cols, c.w_rows, c.w_count, c.ld_w, c.stride_w, BM, true)) return rc;
        if (int rc = make_map_f8(c.what, &mx, c.x, c.x_cols, c.x_rows, 1, c.ld_x, 0, 128, false)) return rc;
        if (int rc = make_map_f8(c.what, &mx32, c.x, c.x_cols, c.x_rows, 1, c.ld_x, 0, 32, false)) return rc;
    }
    // operand types, which dimension is contiguous, scales as powers of two, rows of the tile
    p.idesc = (uint32_t)c.w_type << 7 | (uint32_t)c.x_type << 10 | (MODE != FORWARD ? 1u : 0u) << 15 | (MODE == WGRAD ? 1u : 0u) << 16 | 1u << 23 |
              (uint32_t)((BM * CTAS) >> 7) << 27;
    const int64_t workers = tiles < sm_count() / CTAS ? tiles : sm_count() / CTAS;
    profile_before(st);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(workers * CTAS)); cfg.blockDim = dim3(F8_THREADS); cfg.dynamicSmemBytes = S::TOTAL; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    unsigned na = 0;
    if (CTAS > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = CTAS; attr[na].val.clusterDim.y = 1; attr[na].val.clusterDim.z = 1;
        ++na;
    }
    if (pdl_enabled()) {
        attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[na].val.programmaticStreamSerializationAllowed = 1;
        ++na;
    }
    cfg.attrs = attr; cfg.numAttrs = na;
    QNN_CUDA(cudaLaunchKernelEx(&cfg, kern, mw, mx, mx32, p));
    profile_after(st);
    return check_launch(c.what);
}

template <int MODE, typename TOUT>
int run_f8_typed(const F8Call &c, const F8Params &p, cudaStream_t st)
{
    if constexpr (MODE == WGRAD) {
        return launch_f8<240, MODE, 1, TOUT>(c, p, st);
    } else {
        const int64_t avg = p.M / p.groups;
        if (avg <= 32) return launch_f8<32, MODE, 1, TOUT>(c, p, st);
        if (avg <= 64) return launch_f8<64, MODE, 1, TOUT>(c, p, st);
        if (avg <= 128) return launch_f8<128, MODE, 1, TOUT>(c, p, st);
        return launch_f8<240, MODE, 1, TOUT>(c, p, st);
    }
}
template <int MODE>
int run_f8(const F8Call &c, const F8Params &p, int out_type, cudaStream_t st)
{
    switch (out_type) {
        case QNN_TYPE_F32: return run_f8_typed<MODE, float>(c, p, st);
        case QNN_TYPE_BF16: return run_f8_typed<MODE, __nv_bfloat16>(c, p, st);
        default: return run_f8_typed<MODE, __half>(c, p, st);
    }
}

bool f8_type_ok(int t) { return t == QNN_F8_E4M3 || t == QNN_F8_E5M2; }

int check_operand(const char *what, const char *name, const void *codes, int64_t ld, const void *scale, int64_t ld_scale, int64_t cols, int64_t scale_cols)
{
    QNN_REQUIRE(codes && scale, QNN_ERR_INVALID_ARG, "%s: NULL pointer (%s)", what, name);
    QNN_REQUIRE(ld >= cols, QNN_ERR_INVALID_ARG, "%s: leading dimension of %s below its row length", what, name);
    QNN_REQUIRE(ld_scale >= scale_cols, QNN_ERR_INVALID_ARG, "%s: leading dimension of the scales of %s below their row length", what, name);
    QNN_REQUIRE(aligned(codes, 16) && ld % 16 == 0, QNN_ERR_ALIGNMENT, "%s: codes of %s must be 16-byte aligned, their leading dimension a multiple of 16",
                what, name);
    QNN_REQUIRE(aligned(scale, 16) && ld_scale % 16 == 0, QNN_ERR_ALIGNMENT,
                "%s: scales of %s must be 16-byte aligned, their leading dimension a multiple of 16", what, name);
    QNN_REQUIRE(ld < (int64_t)1 << 40, QNN_ERR_UNSUPPORTED, "%s: leading dimension of %s of 2^40 and more", what, name);
    return QNN_OK;
}

int gemm_f8(const char *what, const void *a, int a_type, int64_t lda, const void *a_scale, int64_t ld_as, const void *b, int b_type, int64_t ldb,
            const void *b_scale, int64_t ld_bs, int across, const float *bias, const int64_t *offsets, int64_t groups, int64_t M, int64_t N, int64_t K,
            void *out, int out_type, int64_t ldo, void *stream)
{
    QNN_REQUIRE(type_ok(out_type), QNN_ERR_INVALID_ARG, "%s: unknown output type %d", what, out_type);
    QNN_REQUIRE(f8_type_ok(a_type) && f8_type_ok(b_type), QNN_ERR_INVALID_ARG, "%s: unknown type of codes", what);
    QNN_REQUIRE(M >= 0 && N >= 0 && K >= 0 && groups >= 0, QNN_ERR_INVALID_ARG, "%s: negative size", what);
    QNN_REQUIRE(across == 0 || across == 1, QNN_ERR_INVALID_ARG, "%s: b_transposed is neither 0 nor 1", what);
    QNN_REQUIRE(M <= (int64_t)1 << 30 && N <= (int64_t)1 << 30 && K <= (int64_t)1 << 30, QNN_ERR_UNSUPPORTED, "%s: a size above 2^30", what);
    QNN_REQUIRE(groups <= MAX_GROUPS, QNN_ERR_UNSUPPORTED, "%s: more than %d groups", what, MAX_GROUPS);
    if (M == 0 || N == 0 || groups == 0) return QNN_OK;
    QNN_REQUIRE(out, QNN_ERR_INVALID_ARG, "%s: NULL pointer", what);
    QNN_REQUIRE(ldo >= N, QNN_ERR_INVALID_ARG, "%s: ldo below N", what);
    QNN_REQUIRE(aligned(out, (size_t)type_bytes(out_type)) && aligned(bias, 4) && aligned(offsets, 8), QNN_ERR_ALIGNMENT,
                "%s: a pointer is not aligned to its elements", what);
    const int64_t kb = ceil_div(K, 128), nb = ceil_div(N, 128);
    if (K > 0) {
        if (int rc = check_operand(what, "a", a, lda, a_scale, ld_as, K, kb)) return rc;
        if (int rc = check_operand(what, "b", b, ldb, b_scale, ld_bs, across ? N : K, across ? nb : kb)) return rc;
    }
    F8Params p{};
    p.M = M; p.N = (int32_t)N; p.nkb = (int32_t)kb; p.groups = (int32_t)groups;
    p.offsets = offsets;
    p.w_scale = static_cast<const uint8_t *>(b_scale); p.ld_ws = ld_bs; p.stride_ws = (across ? kb : nb) * ld_bs;
    p.x_scale = static_cast<const uint8_t *>(a_scale); p.ld_xs = ld_as;
    p.bias = bias; p.out = out; p.ldo = ldo;
    p.vec_out = aligned(out, 16) && ldo * type_bytes(out_type) % 16 == 0;
    const int64_t rows = across ? K : N, cols = across ? N : K;
    QNN_REQUIRE(K == 0 || groups == 1 || ldb <= (((int64_t)1 << 40) - 1) / rows, QNN_ERR_UNSUPPORTED, "%s: matrices of b of 2^40 bytes and more", what);
    const F8Call c = {what, b, b_type, rows, cols, ldb, groups == 1 ? ldb : rows * ldb, (int32_t)groups, a, a_type, M, K, lda};
    return across ? run_f8<ACROSS>(c, p, out_type, as_stream(stream)) : run_f8<FORWARD>(c, p, out_type, as_stream(stream));
}

}  // namespace

int gemm_f8_status(int *code)
{
    QNN_CUDA(status_read_clear(code));
    return QNN_OK;
}

}  // namespace qnn

using namespace qnn;

extern "C" {

int qnn_gemm_f8(const void *a, int a_type, int64_t lda, const void *a_scale, int64_t ld_as, const void *b, int b_type, int64_t ldb, const void *b_scale,
                int64_t ld_bs, int b_transposed, const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_type, int64_t ldo, void *stream)
{
    return gemm_f8("qnn_gemm_f8", a, a_type, lda, a_scale, ld_as, b, b_type, ldb, b_scale, ld_bs, b_transposed, bias, nullptr, 1, M, N, K, out, out_type,
                   ldo, stream);
}

int qnn_gemm_f8_grouped(const void *a, int a_type, int64_t lda, const void *a_scale, int64_t ld_as, const void *b, int b_type, int64_t ldb,
                        const void *b_scale, int64_t ld_bs, int b_transposed, const float *bias, const int64_t *offsets, int64_t groups, int64_t M,
                        int64_t N, int64_t K, void *out, int out_type, int64_t ldo, void *stream)
{
    const char *what = "qnn_gemm_f8_grouped";
    QNN_REQUIRE(offsets || M == 0 || N == 0 || groups == 0, QNN_ERR_INVALID_ARG, "%s: offsets are NULL", what);
    return gemm_f8(what, a, a_type, lda, a_scale, ld_as, b, b_type, ldb, b_scale, ld_bs, b_transposed, bias, offsets, groups, M, N, K, out, out_type, ldo,
                   stream);
}

int qnn_gemm_f8_wgrad(const void *dy, int dy_type, int64_t ld_dy, const void *dy_scale, int64_t ld_dys, const void *x, int x_type, int64_t ldx,
                      const void *x_scale, int64_t ld_xs, const int64_t *offsets, int64_t groups, int64_t M, int64_t N, int64_t K, void *dw, int dw_type,
                      int64_t ld_dw, void *stream)
{
    const char *what = "qnn_gemm_f8_wgrad";
    QNN_REQUIRE(type_ok(dw_type), QNN_ERR_INVALID_ARG, "%s: unknown output type %d", what, dw_type);
    QNN_REQUIRE(f8_type_ok(dy_type) && f8_type_ok(x_type), QNN_ERR_INVALID_ARG, "%s: unknown type of codes", what);
    QNN_REQUIRE(M >= 0 && N >= 0 && K >= 0 && groups >= 0, QNN_ERR_INVALID_ARG, "%s: negative size", what);
    QNN_REQUIRE(M <= (int64_t)1 << 30 && N <= (int64_t)1 << 30 && K <= (int64_t)1 << 30, QNN_ERR_UNSUPPORTED, "%s: a size above 2^30", what);
    QNN_REQUIRE(groups <= MAX_GROUPS, QNN_ERR_UNSUPPORTED, "%s: more than %d groups", what, MAX_GROUPS);
    if (N == 0 || K == 0 || groups == 0) return QNN_OK;
    QNN_REQUIRE(dw && (offsets || groups == 1), QNN_ERR_INVALID_ARG, "%s: NULL pointer", what);
    QNN_REQUIRE(ld_dw >= K, QNN_ERR_INVALID_ARG, "%s: ld_dw below K", what);
    QNN_REQUIRE(aligned(dw, (size_t)type_bytes(dw_type)) && aligned(offsets, 8), QNN_ERR_ALIGNMENT, "%s: a pointer is not aligned to its elements", what);
    if (M > 0) {
        if (int rc = check_operand(what, "dy", dy, ld_dy, dy_scale, ld_dys, N, N)) return rc;
        if (int rc = check_operand(what, "x", x, ldx, x_scale, ld_xs, K, K)) return rc;
    }
    F8Params p{};
    p.M = M; p.N = (int32_t)N; p.C = (int32_t)K; p.groups = (int32_t)groups;
    p.offsets = offsets;
    p.w_scale = static_cast<const uint8_t *>(dy_scale); p.ld_ws = ld_dys;
    p.x_scale = static_cast<const uint8_t *>(x_scale); p.ld_xs = ld_xs;
    p.out = dw; p.ldo = ld_dw;
    p.vec_out = aligned(dw, 16) && ld_dw * type_bytes(dw_type) % 16 == 0;
    const int64_t rows = M > 0 ? 128 * (M / 128 + groups) : 0;          // rows of all blocks, at most
    const F8Call c = {what, dy, dy_type, rows, N, ld_dy, ld_dy, 1, x, x_type, rows, K, ldx};
    return run_f8<WGRAD>(c, p, dw_type, as_stream(stream));
}

}  // extern "C"
